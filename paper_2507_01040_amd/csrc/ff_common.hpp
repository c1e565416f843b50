// Shared parts of the feed-forward operators (cliffconv_ff.h): types, the
// pointwise activations, the dropout generator, and what their launchers take.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cliffconv_ff.h"
#include "common.hpp"

namespace cliff {

// What the kernels know of a dropout: element (r, c) is dropped where its
// word of the generator is at most `last` (round(p 2^32) - 1).
struct DropArgs {
    const int64_t* rng;  // NULL: no dropout
    uint32_t last;
    float scale;
};

struct DenseArgs {
    int64_t M, K, N;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    int w_out_in;
    const void* bias;
    int act;
    DropArgs drop;
    const void* residual;
    int64_t ldr;
    void* pre;
    int64_t ldp;
    void* y;
    int64_t ldy;
    void* workspace;
};

struct DenseBackwardArgs {
    int64_t M, K, N;
    const void* dy;
    int64_t lddy;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    int w_out_in;
    const void* pre;
    int64_t ldp;
    int act;
    DropArgs drop;
    void* dx;
    int64_t lddx;
    void* dw;
    int64_t lddw;
    void* dbias;
    void* workspace;
};

struct NormArgs {
    int64_t rows, d;
    const void* x;
    int64_t ldx;
    const void* weight;
    const void* bias;
    float eps;
    void* y;
    int64_t ldy;
    float* mean;
    float* rstd;
};

struct NormBackwardArgs {
    int64_t rows, d;
    const void* dy;
    int64_t lddy;
    const void* x;
    int64_t ldx;
    const float* mean;
    const float* rstd;
    const void* weight;
    const void* dresidual;
    int64_t ldr;
    void* dx;
    int64_t lddx;
    void* dweight;
    void* dbias;
    void* workspace;
};

struct DropoutArgs {
    int64_t rows, d;
    const void* x;
    int64_t ldx;
    DropArgs drop;
    const void* residual;
    int64_t ldr;
    void* y;
    int64_t ldy;
};

// Launchers (the arguments are checked): dtype is a cliff_dtype.
cliff_status launch_dense(int dtype, const DenseArgs& a, hipStream_t stream);
int64_t dense_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status launch_dense_backward(int dtype, const DenseBackwardArgs& a, hipStream_t stream);
int64_t dense_backward_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status launch_layer_norm(int dtype, const NormArgs& a, hipStream_t stream);
cliff_status launch_layer_norm_backward(int dtype, const NormBackwardArgs& a, hipStream_t stream);
int64_t layer_norm_backward_workspace(int dtype, int64_t rows, int64_t d);
cliff_status launch_dropout(int dtype, const DropoutArgs& a, hipStream_t stream);

inline cliff_status launched()
{
    return hipGetLastError() == hipSuccess ? CLIFF_OK : CLIFF_EDEVICE;
}

// Calls f with a value of the element type of `dtype`.
template <typename F>
cliff_status with_type(int dtype, F f)
{
    switch (dtype) {
    case CLIFF_F32: return f(float{});
    case CLIFF_BF16: return f(__bf16{});
    case CLIFF_F16: return f(_Float16{});
    }
    return CLIFF_EINVAL;
}

// The four words of Philox4x32-7 for elements 4 q to 4 q + 3 of row r.
// Seven rounds are the fewest that its authors found to pass every test of
// theirs; a round is two 32 x 32 -> 64 products.
struct Words {
    uint32_t w[4];
};
__host__ __device__ inline Words philox(uint64_t key, uint32_t step, uint32_t q, int64_t r)
{
    uint32_t c0 = q, c1 = (uint32_t)r, c2 = (uint32_t)((uint64_t)r >> 32), c3 = step;
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

__device__ inline float gelu_cdf(float v)  // Phi(v)
{
    return 0.5f * (1.0f + erff(v * 0.70710678118654752f));
}

__device__ inline float activate(int act, float v)
{
    switch (act) {
    case CLIFF_ACT_RELU: return v > 0.f ? v : 0.f;
    case CLIFF_ACT_GELU: return v * gelu_cdf(v);
    case CLIFF_ACT_SILU: return v / (1.0f + __expf(-v));
    }
    return v;
}

__device__ inline float activate_slope(int act, float v)
{
    switch (act) {
    case CLIFF_ACT_RELU: return v > 0.f ? 1.f : 0.f;
    case CLIFF_ACT_GELU: return gelu_cdf(v) + v * 0.39894228040143268f * __expf(-0.5f * v * v);
    case CLIFF_ACT_SILU: {
        const float s = 1.0f / (1.0f + __expf(-v));
        return s * (1.0f + v * (1.0f - s));
    }
    }
    return 1.f;
}

}  // namespace cliff
