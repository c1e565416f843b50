// Parts of the kernels that go over rows (layer norm, dropout): 16 bytes of a
// row at a time, and sums over the lanes of a wave.
#pragma once

#include "ff_common.hpp"

namespace cliff {

template <typename T>
__device__ inline void unpack16(const raw16& r, float* v)
{
    constexpr int E = per16<T>;
    typedef T vt __attribute__((ext_vector_type(E)));
    const vt t = __builtin_bit_cast(vt, r);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)t[e];
}

template <typename T>
__device__ inline void store16(T* p, const float* v, int have)
{
    constexpr int E = per16<T>;
    typedef T vt __attribute__((ext_vector_type(E)));
    typedef float vf __attribute__((ext_vector_type(E)));
    vf f;
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = v[e];
    const vt t = __builtin_convertvector(f, vt);
    if (have >= E) {
        __builtin_memcpy(p, &t, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < have) p[e] = t[e];
    }
}

template <int CTRL>
__device__ inline float dpp(float v)
{
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// The sum of v over each aligned group of N lanes, in every one of them.
template <int N>
__device__ inline float lane_sum(float v)
{
    static_assert(N == 16 || N == 64, "lanes");
    v += dpp<0xb1>(v);   // neighbours
    v += dpp<0x4e>(v);   // pairs
    v += dpp<0x141>(v);  // halves of 8, mirrored
    v += dpp<0x140>(v);  // halves of 16, mirrored
    if constexpr (N == 64) {
        const uint32_t a = __builtin_bit_cast(uint32_t, v);
        const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
        const uint32_t s0 = s[0], s1 = s[1];
        v = __builtin_bit_cast(float, s0) + __builtin_bit_cast(float, s1);
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto t = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const uint32_t t0 = t[0], t1 = t[1];
        v = __builtin_bit_cast(float, t0) + __builtin_bit_cast(float, t1);
    }
    return v;
}

// The sums of v[0..R) over the TPR threads of a row, in every one of them: 16
// or 64 lanes, or the whole workgroup of TPR threads (then through `lds`, R
// floats a wave, with one barrier; the caller alternates two of them).
template <int TPR, int R>
__device__ inline void row_sums(float (&v)[R], float* lds)
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = lane_sum<(TPR < 64 ? 16 : 64)>(v[r]);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) lds[(threadIdx.x >> 6) * R + r] = v[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            v[r] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[r] += lds[w * R + r];
        }
    }
}

}  // namespace cliff
