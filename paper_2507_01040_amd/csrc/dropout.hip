// Dropout of a matrix of rows, with an optional residual: y = residual +
// dropout(x).  The mask comes from a counter (ff_common.hpp), so the gradient
// is the same call on the gradient and nothing is stored.
//
// Bound by memory, with the generator close behind: 7 rounds of two 32 x 32 ->
// 64 products for four elements.  A thread takes 16 bytes of each of ROWS rows,
// all loads before the first round; groups of four columns never span two
// threads, so no word is formed twice.  16384 x 4096 bf16 with a residual 74 us
// (5.4 TB/s); 1001 x 777 fp32 3.9 us, a launch.
#include <stdio.h>

#include <algorithm>

#include "rows.hpp"

namespace cliff {
namespace {

constexpr int ROWS = 4;

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, uint32_t pieces, int64_t n)
{
    constexpr int E = per16<T>;
    const int64_t i = workgroup_id() * 256ll + threadIdx.x;
    if (i >= n) return;
    const int64_t g = n >> 32 ? i / pieces : (int64_t)((uint32_t)i / pieces), r0 = g * ROWS;
    const int col = (int)(i - g * pieces) * E, have = (int)a.d - col;
    uint64_t key = 0;
    uint32_t step = 0;
    if (a.drop.rng) {
        key = (uint64_t)a.drop.rng[0];
        step = (uint32_t)a.drop.rng[1];
    }
    raw16 x[ROWS], res[ROWS];
    auto piece = [&](const void* from, int64_t ld, int r) {
        const int64_t row = r0 + r < a.rows ? r0 + r : a.rows - 1;
        const T* const line = static_cast<const T*>(from) + row * ld;
        return a.d < E ? load16_narrow(line, col, a.d) : load16(line, col, a.d);
    };
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        x[r] = piece(a.x, a.ldx, r);
        if (a.residual) res[r] = piece(a.residual, a.ldr, r);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float v[E], u[E];
        if (a.d >= E) settle16<T>(x[r], col, a.d);
        unpack16<T>(x[r], v);
        if (a.drop.rng)
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                const Words w = philox(key, step, (uint32_t)(col / 4 + q), r0 + r);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[4 * q + e] = w.w[e] <= a.drop.last ? 0.f : v[4 * q + e] * a.drop.scale;
            }
        if (a.residual) {
            if (a.d >= E) settle16<T>(res[r], col, a.d);
            unpack16<T>(res[r], u);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += u[e];
        }
        if (r0 + r < a.rows) store16(static_cast<T*>(a.y) + (r0 + r) * a.ldy + col, v, have);
    }
}

}  // namespace

cliff_status launch_dropout(int dtype, const DropoutArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t pieces = (a.d + per16<T> - 1) / per16<T>;
        const int64_t n = pieces * ((a.rows + ROWS - 1) / ROWS), blocks = (n + 255) / 256;
        if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
        if (debug_enabled())
            fprintf(stderr, "cliffconv: dropout %lld x %lld, %lld workgroups\n", (long long)a.rows, (long long)a.d,
                    (long long)blocks);
        hipLaunchKernelGGL(dropout_kernel<T>, grid_of(blocks), dim3(256), 0, stream, a, (uint32_t)pieces, n);
        return launched();
    });
}

}  // namespace cliff
