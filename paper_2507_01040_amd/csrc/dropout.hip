// Dropout of a matrix of rows, with an optional residual: y = residual +
// dropout(x).  The mask comes from a counter (ff_common.hpp), so the gradient
// is the same call on the gradient and nothing is stored.
#include <stdio.h>

#include <algorithm>

#include "ff_common.hpp"

namespace cliff {
namespace {

// One thread per group of four columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a)
{
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.residual);
    T* y = static_cast<T*>(a.y);
    const int64_t nq = (a.d + 3) / 4, n = a.rows * nq;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        const int64_t r = i / nq, q = i % nq;
        Words w{};
        if (a.drop.rng) w = philox((uint64_t)a.drop.rng[0], (uint32_t)a.drop.rng[1], (uint32_t)q, r);
        for (int e = 0; e < 4; ++e) {
            const int64_t c = 4 * q + e;
            if (c >= a.d) break;
            float v = (float)x[r * a.ldx + c] * a.drop.scale;
            if (a.drop.rng && w.w[e] <= a.drop.last) v = 0.f;
            if (res) v += (float)res[r * a.ldr + c];
            y[r * a.ldy + c] = (T)v;
        }
    }
}

}  // namespace

cliff_status launch_dropout(int dtype, const DropoutArgs& a, hipStream_t stream)
{
    const int64_t n = a.rows * ((a.d + 3) / 4);
    const int64_t blocks = std::min<int64_t>((n + 255) / 256, 1 << 20);
    if (debug_enabled())
        fprintf(stderr, "cliffconv: dropout type %d, %lld x %lld, %lld workgroups\n", dtype,
                (long long)a.rows, (long long)a.d, (long long)blocks);
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        hipLaunchKernelGGL(dropout_kernel<decltype(t)>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
        return launched();
    });
}

}  // namespace cliff
