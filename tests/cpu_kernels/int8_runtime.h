// What the 8-bit kernels use of HIP's device language beside hip_runtime.h (test
// infrastructure; see block_main.cpp): matrix instructions of 8-bit integers, with
// the lanes' layout of those of 16 bits.
#pragma once

#include <hip/hip_runtime.h>

namespace emulate {

void wait_loads_but(int n);

enum { MFMA_I8 = TR16 + 1 };

template <int S, typename V, typename Acc>
struct ProductI8 {
    struct In {
        V a, b;
        Acc c;
    };
    static void f(const In* in, Acc* out)
    {
        constexpr int E = 16, K = E * WAVE / S;
        int a[S][K], b[K][S];
        for (int l = 0; l < WAVE; ++l) {
            int8_t va[E], vb[E];
            memcpy(va, &in[l].a, E);
            memcpy(vb, &in[l].b, E);
            for (int e = 0; e < E; ++e) {
                a[l % S][E * (l / S) + e] = va[e];
                b[E * (l / S) + e][l % S] = vb[e];
            }
        }
        for (int i = 0; i < S; ++i) {
            const int e = S == 32 ? i / 8 * 4 + i % 4 : i % 4, h = S == 32 ? i / 4 % 2 : i / 4;
            for (int j = 0; j < S; ++j) {
                int d = in[S * h + j].c[e];
                for (int k = 0; k < K; ++k) d += a[i][k] * b[k][j];
                out[S * h + j][e] = d;
            }
        }
    }
};
template <int S, typename V, typename Acc>
Acc mfma_i8(const V& a, const V& b, const Acc& c)
{
    typedef ProductI8<S, V, Acc> P;
    return together<MFMA_I8, typename P::In, Acc, P::f>(typename P::In{a, b, c});
}

// Byte i of the result is byte selector_i of (a, b), a's bytes being 4 to 7; selector
// 0x0c gives zero.
inline uint32_t perm(uint32_t a, uint32_t b, uint32_t selector)
{
    const uint64_t both = (uint64_t)a << 32 | b;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = selector >> 8 * i & 0xff;
        if (s < 8) r |= (uint32_t)(both >> 8 * s & 0xff) << 8 * i;
    }
    return r;
}

}  // namespace emulate

#define __builtin_amdgcn_perm emulate::perm
#define __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, x, y, z) emulate::mfma_i8<32>(a, b, c)
#define __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, x, y, z) emulate::mfma_i8<16>(a, b, c)
