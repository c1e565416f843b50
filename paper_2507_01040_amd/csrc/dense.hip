// Dense layer with its epilogue, and its gradient.
#include <stdio.h>

#include <algorithm>

#include "ff_common.hpp"

namespace cliff {
namespace {

// C[m, n] = sum_k A(m, k) B(k, n), operands by two strides each.
struct ProductArgs {
    int64_t M, K, N;
    const void* a;
    int64_t am, ak;
    const void* b;
    int64_t bk, bn;
    // epilogue
    const void* bias;
    int act;
    DropArgs drop;
    const void* residual;
    int64_t ldr;
    void* pre;
    int64_t ldp;
    void* y;
    int64_t ldy;
};

// 32 x 32 outputs per workgroup, one per thread in four passes.
template <typename T>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs p)
{
    __shared__ float as[32][33], bs[32][33];
    const int64_t tn = (p.N + 31) / 32;
    const int64_t m0 = blockIdx.x / tn * 32, n0 = blockIdx.x % tn * 32;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    float acc[4] = {};
    for (int64_t k0 = 0; k0 < p.K; k0 += 32) {
        for (int i = 0; i < 4; ++i) {
            const int row = ty + 8 * i;
            const int64_t m = m0 + row, k = k0 + tx, kb = k0 + row, n = n0 + tx;
            as[row][tx] = m < p.M && k < p.K ? (float)static_cast<const T*>(p.a)[m * p.am + k * p.ak] : 0.f;
            bs[row][tx] = kb < p.K && n < p.N ? (float)static_cast<const T*>(p.b)[kb * p.bk + n * p.bn] : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 32; ++k)
            for (int i = 0; i < 4; ++i) acc[i] += as[ty + 8 * i][k] * bs[k][tx];
        __syncthreads();
    }
    const int64_t n = n0 + tx;
    if (n >= p.N) return;
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + ty + 8 * i;
        if (m >= p.M) continue;
        float v = acc[i] + (p.bias ? (float)static_cast<const T*>(p.bias)[n] : 0.f);
        if (p.pre) static_cast<T*>(p.pre)[m * p.ldp + n] = (T)v;
        v = activate(p.act, v);
        if (p.drop.rng) {
            const Words w = philox((uint64_t)p.drop.rng[0], (uint32_t)p.drop.rng[1], (uint32_t)(n >> 2), m);
            v = w.w[n & 3] <= p.drop.last ? 0.f : v * p.drop.scale;
        }
        if (p.residual) v += (float)static_cast<const T*>(p.residual)[m * p.ldr + n];
        static_cast<T*>(p.y)[m * p.ldy + n] = (T)v;
    }
}

// g = dropout(dy) f'(pre) into the workspace [M, N].
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(DenseBackwardArgs a, T* g)
{
    const int64_t n = a.M * a.N;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        const int64_t r = i / a.N, c = i % a.N;
        float v = (float)static_cast<const T*>(a.dy)[r * a.lddy + c];
        if (a.act != CLIFF_ACT_NONE)
            v *= activate_slope(a.act, (float)static_cast<const T*>(a.pre)[r * a.ldp + c]);
        if (a.drop.rng) {
            const Words w = philox((uint64_t)a.drop.rng[0], (uint32_t)a.drop.rng[1], (uint32_t)(c >> 2), r);
            v = w.w[c & 3] <= a.drop.last ? 0.f : v * a.drop.scale;
        }
        g[i] = (T)v;
    }
}

template <typename T>
__global__ __launch_bounds__(64) void bias_kernel(DenseBackwardArgs a)
{
    const int64_t c = blockIdx.x;
    float t = 0.f;
    for (int64_t r = threadIdx.x; r < a.M; r += 64) {
        float v = (float)static_cast<const T*>(a.dy)[r * a.lddy + c];
        if (a.act != CLIFF_ACT_NONE)
            v *= activate_slope(a.act, (float)static_cast<const T*>(a.pre)[r * a.ldp + c]);
        if (a.drop.rng) {
            const Words w = philox((uint64_t)a.drop.rng[0], (uint32_t)a.drop.rng[1], (uint32_t)(c >> 2), r);
            v = w.w[c & 3] <= a.drop.last ? 0.f : v * a.drop.scale;
        }
        t += v;
    }
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if (threadIdx.x == 0) static_cast<T*>(a.dbias)[c] = (T)t;
}

template <typename T>
cliff_status product(const ProductArgs& p, hipStream_t stream)
{
    const int64_t blocks = (p.M + 31) / 32 * ((p.N + 31) / 32);
    if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    hipLaunchKernelGGL(product_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    return launched();
}

}  // namespace

int64_t dense_workspace(int, int64_t, int64_t, int64_t) { return 0; }
int64_t dense_backward_workspace(int dtype, int64_t M, int64_t, int64_t N)
{
    return (M * N * (dtype == CLIFF_F32 ? 4 : 2) + 15) / 16 * 16;
}

cliff_status launch_dense(int dtype, const DenseArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        ProductArgs p{a.M, a.K, a.N, a.x, a.ldx, 1, a.w, a.w_out_in ? 1 : a.ldw, a.w_out_in ? a.ldw : 1,
                      a.bias, a.act, a.drop, a.residual, a.ldr, a.pre, a.ldp, a.y, a.ldy};
        return product<decltype(t)>(p, stream);
    });
}

cliff_status launch_dense_backward(int dtype, const DenseBackwardArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const void* g = a.dy;
        int64_t ldg = a.lddy;
        if (a.M && (a.act != CLIFF_ACT_NONE || a.drop.rng)) {
            T* gw = static_cast<T*>(a.workspace);
            const int64_t blocks = std::min<int64_t>((a.M * a.N + 255) / 256, 1 << 20);
            hipLaunchKernelGGL(slope_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, stream, a, gw);
            g = gw;
            ldg = a.N;
        }
        cliff_status s = CLIFF_OK;
        const DropArgs none{nullptr, 0, 1.f};
        if (a.dbias) {
            hipLaunchKernelGGL(bias_kernel<T>, dim3((unsigned)a.N), dim3(64), 0, stream, a);
            s = launched();
        }
        if (s == CLIFF_OK && a.dx && a.M) {
            ProductArgs p{a.M, a.N, a.K, g, ldg, 1, a.w, a.w_out_in ? a.ldw : 1, a.w_out_in ? 1 : a.ldw,
                          nullptr, CLIFF_ACT_NONE, none, nullptr, 0, nullptr, 0, a.dx, a.lddx};
            s = product<T>(p, stream);
        }
        if (s == CLIFF_OK && a.dw) {
            // in the order of w: [K, N] = x^T g or [N, K] = g^T x
            ProductArgs p{a.K, a.M, a.N, a.x, 1, a.ldx, g, ldg, 1, nullptr, CLIFF_ACT_NONE, none, nullptr, 0,
                          nullptr, 0, a.dw, a.lddw};
            if (a.w_out_in) {
                std::swap(p.M, p.N);
                p.a = g;
                p.ak = ldg;
                p.b = a.x;
                p.bk = a.ldx;
            }
            s = product<T>(p, stream);
        }
        return s;
    });
}

}  // namespace cliff
