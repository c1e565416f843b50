// Layer norm over the columns of rows, forward and backward.
#include <stdio.h>

#include <algorithm>

#include "ff_common.hpp"

namespace cliff {
namespace {

constexpr int NORM_THREADS = 256;

// The sum of v over the workgroup, in every thread.
__device__ inline float block_sum(float v, float* s)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
    for (int i = 0; i < NORM_THREADS / 64; ++i) t += s[i];
    return t;
}

// One workgroup per row at a time.
template <typename T>
__global__ __launch_bounds__(NORM_THREADS) void norm_kernel(NormArgs a)
{
    __shared__ float s[NORM_THREADS / 64];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        T* y = static_cast<T*>(a.y) + r * a.ldy;
        float t = 0.f;
        for (int64_t c = threadIdx.x; c < a.d; c += NORM_THREADS) t += (float)x[c];
        const float mean = block_sum(t, s) / (float)a.d;
        t = 0.f;
        for (int64_t c = threadIdx.x; c < a.d; c += NORM_THREADS) {
            const float v = (float)x[c] - mean;
            t += v * v;
        }
        const float rstd = 1.0f / sqrtf(block_sum(t, s) / (float)a.d + a.eps);
        for (int64_t c = threadIdx.x; c < a.d; c += NORM_THREADS) {
            float v = ((float)x[c] - mean) * rstd;
            if (a.weight) v *= (float)static_cast<const T*>(a.weight)[c];
            if (a.bias) v += (float)static_cast<const T*>(a.bias)[c];
            y[c] = (T)v;
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(NORM_THREADS) void norm_dx_kernel(NormBackwardArgs a)
{
    __shared__ float s[NORM_THREADS / 64];
    const T* w = static_cast<const T*>(a.weight);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* res = static_cast<const T*>(a.dresidual) + r * a.ldr;
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float t0 = 0.f, t1 = 0.f;
        for (int64_t c = threadIdx.x; c < a.d; c += NORM_THREADS) {
            const float q = (float)dy[c] * (w ? (float)w[c] : 1.f);
            t0 += q;
            t1 += q * ((float)x[c] - mean) * rstd;
        }
        t0 = block_sum(t0, s) / (float)a.d;
        t1 = block_sum(t1, s) / (float)a.d;
        for (int64_t c = threadIdx.x; c < a.d; c += NORM_THREADS) {
            const float q = (float)dy[c] * (w ? (float)w[c] : 1.f);
            float v = rstd * (q - t0 - ((float)x[c] - mean) * rstd * t1);
            if (a.dresidual) v += (float)res[c];
            dx[c] = (T)v;
        }
    }
}

// The weight's and bias's gradients: workgroup (column block, part) sums its
// share of the rows for 256 columns into the workspace [part][2][d] ...
template <typename T>
__global__ __launch_bounds__(NORM_THREADS) void norm_dw_kernel(NormBackwardArgs a, int64_t rows_per_part)
{
    const int64_t c = blockIdx.x * (int64_t)NORM_THREADS + threadIdx.x;
    if (c >= a.d) return;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float t0 = 0.f, t1 = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float g = (float)static_cast<const T*>(a.dy)[r * a.lddy + c];
        t0 += g * ((float)static_cast<const T*>(a.x)[r * a.ldx + c] - a.mean[r]) * a.rstd[r];
        t1 += g;
    }
    float* p = static_cast<float*>(a.workspace) + 2 * blockIdx.y * a.d;
    p[c] = t0;
    p[a.d + c] = t1;
}

// ... and this joins the parts in order.
template <typename T>
__global__ __launch_bounds__(NORM_THREADS) void norm_join_kernel(NormBackwardArgs a, int parts)
{
    const int64_t c = blockIdx.x * (int64_t)NORM_THREADS + threadIdx.x;
    if (c >= a.d) return;
    const float* p = static_cast<const float*>(a.workspace);
    float t0 = 0.f, t1 = 0.f;
    for (int i = 0; i < parts; ++i) {
        t0 += p[2 * i * a.d + c];
        t1 += p[(2 * i + 1) * a.d + c];
    }
    if (a.dweight) static_cast<T*>(a.dweight)[c] = (T)t0;
    if (a.dbias) static_cast<T*>(a.dbias)[c] = (T)t1;
}

int norm_parts(int64_t rows, int64_t d)
{
    const int64_t blocks = (d + NORM_THREADS - 1) / NORM_THREADS;
    return (int)std::max<int64_t>(0, std::min<int64_t>({(rows + 31) / 32, 2048 / blocks + 1, 512}));
}

}  // namespace

int64_t layer_norm_backward_workspace(int, int64_t rows, int64_t d)
{
    return 8 * d * norm_parts(rows, d);
}

cliff_status launch_layer_norm(int dtype, const NormArgs& a, hipStream_t stream)
{
    const int64_t blocks = std::min<int64_t>(a.rows, 1 << 20);
    if (debug_enabled())
        fprintf(stderr, "cliffconv: layer_norm type %d, %lld x %lld, %lld workgroups\n", dtype,
                (long long)a.rows, (long long)a.d, (long long)blocks);
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        hipLaunchKernelGGL(norm_kernel<decltype(t)>, dim3((unsigned)blocks), dim3(NORM_THREADS), 0, stream, a);
        return launched();
    });
}

cliff_status launch_layer_norm_backward(int dtype, const NormBackwardArgs& a, hipStream_t stream)
{
    const int64_t blocks = std::min<int64_t>(a.rows, 1 << 20);
    const int parts = norm_parts(a.rows, a.d);
    if (debug_enabled())
        fprintf(stderr, "cliffconv: layer_norm_backward type %d, %lld x %lld, %d parts\n", dtype,
                (long long)a.rows, (long long)a.d, parts);
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const unsigned cols = (unsigned)((a.d + NORM_THREADS - 1) / NORM_THREADS);
        // the sums first: dx may be dy
        if (a.dweight || a.dbias) {
            if (parts)
                hipLaunchKernelGGL(norm_dw_kernel<T>, dim3(cols, parts), dim3(NORM_THREADS), 0, stream, a,
                                   (a.rows + parts - 1) / std::max(parts, 1));
            hipLaunchKernelGGL(norm_join_kernel<T>, dim3(cols), dim3(NORM_THREADS), 0, stream, a, parts);
        }
        if (a.rows)
            hipLaunchKernelGGL(norm_dx_kernel<T>, dim3((unsigned)blocks), dim3(NORM_THREADS), 0, stream, a);
        return launched();
    });
}

}  // namespace cliff
