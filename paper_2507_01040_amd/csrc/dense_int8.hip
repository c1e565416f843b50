// Dense layer of 8-bit integers with a scale for each row and each output:
//   y = residual + f(x_scale w_scale sum(x w) + bias).
// Both operands are contiguous along the contraction; sums are 32-bit integers,
// exact in any order.
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include "dense_geom.hpp"
#include "ff_common.hpp"
#include "lds_load.hpp"
#include "rows.hpp"

namespace cliff {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Sums [m, n] = sum_k a[m, k] b[n, k], and what finishes them.
struct Int8Args {
    int64_t M, N, K;
    const int8_t* a;
    int64_t lda;
    const int8_t* b;
    int64_t ldb;
    const float* a_scale;
    const float* b_scale;
    const void* bias;
    int act;
    const void* residual;
    int64_t ldr;
    void* y;
    int64_t ldy;
};

__device__ inline i16v mma(const u4& x, const u4& y, const i16v& c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i4, x), __builtin_bit_cast(i4, y), c, 0, 0, 0);
}

// What a group of four columns needs besides its sums, loaded early.
struct Ends {
    f4 scale, bias;
};
template <typename T>
__device__ inline Ends load_ends(const Int8Args& p, int64_t n)
{
    Ends e{f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
    if (n >= p.N) return e;
    const int have = p.N - n < 4 ? (int)(p.N - n) : 4;
    e.scale = load4(p.b_scale + n, have);
    if (p.bias) e.bias = load4(static_cast<const T*>(p.bias) + n, have);
    return e;
}

// R rows of a group of four columns: rows m, m + step, ...
template <typename T, int R>
__device__ inline void finish_rows(const Int8Args& p, int64_t m, int step, int64_t n, const i4 (&v)[R], const Ends& e)
{
    const int have = p.N - n >= 4 ? 4 : (int)(p.N - n);
    f4 res[R];
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (m + r * step < p.M) {
            s[r] = p.a_scale[m + r * step];
            if (p.residual) res[r] = load4(static_cast<const T*>(p.residual) + (m + r * step) * p.ldr + n, have);
        }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (m + r * step >= p.M) break;
        f4 u;
        // the smaller scale first: neither product leaves fp32 where the result does
        // not (comparisons keep a NaN)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool less = s[r] < e.scale[i];
            u[i] = fmaf((float)v[r][i] * (less ? s[r] : e.scale[i]), less ? e.scale[i] : s[r], e.bias[i]);
        }
        activate4<sizeof(T) == 4>(p.act, u);
        if (p.residual) u += res[r];
        store4(static_cast<T*>(p.y) + (m + r * step) * p.ldy + n, u, have);
    }
}

// The outputs of a wave's MI x NI blocks of 32 x 32 from row m1, column n1 on: 32
// rows at a time through LDS, so that 16 lanes hold 64 neighbouring columns of a
// row.  Begins with a barrier: the stages there are done with.
constexpr int EW = 64 + 4;  // integers per row there
template <typename T, int MI, int NI>
__device__ inline void write_tile(const Int8Args& p, int64_t m1, int64_t n1, const i16v (&acc)[MI][NI], char* smem,
                                  int lane, int wave)
{
    const int64_t n = n1 + 4 * (lane & 15);
    const Ends ends = load_ends<T>(p, n);
    __syncthreads();
    int* const tile = reinterpret_cast<int*>(smem) + wave * 32 * EW;
    auto put = [&](const i16v& c, int j) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<i4*>(tile + (lane & 31) * EW + 32 * j + 8 * g + 4 * (lane >> 5)) =
                i4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
    };
    static_assert(MI <= 4 && NI == 2, "blocks");
#pragma unroll 1
    for (int i = 0; i < MI; ++i) {  // not unrolled: one copy of what follows the switch
        switch (i) {
        case 0: put(acc[0][0], 0); put(acc[0][1], 1); break;
        case 1: if constexpr (MI > 1) { put(acc[1][0], 0); put(acc[1][1], 1); } break;
        case 2: if constexpr (MI > 2) { put(acc[2][0], 0); put(acc[2][1], 1); } break;
        case 3: if constexpr (MI > 3) { put(acc[3][0], 0); put(acc[3][1], 1); } break;
        }
        wave_fence();
        if (n < p.N) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int r0 = 16 * h + (lane >> 4);
                i4 v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const i4*>(tile + (r0 + 4 * r) * EW + 4 * (lane & 15));
                finish_rows<T, 4>(p, m1 + 32 * i + r0, 4, n, v, ends);
            }
        }
        wave_fence();
    }
}

// 128 x 128 outputs per workgroup of 2 x 2 waves, stages of 128 contraction values
// (slots of 16, as of 8 in 16 bits), of any alignment, one stage ahead in registers.
constexpr int TILE = 128, KT = 128;
template <typename T>
__global__ __launch_bounds__(256) void int8_tile_kernel(Int8Args p)
{
    constexpr int NT = 256, MI = 2, NI = 2;
    constexpr Stage S{TILE, KT / 2, true};
    constexpr int L = S.slots() / NT, KK = KT / 32;
    __shared__ __align__(16) char smem[2 * S.bytes() > 4 * 32 * EW * 4 ? 2 * S.bytes() : 4 * 32 * EW * 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2 * 64, wn = wave % 2 * 64;
    const uint32_t tm = (uint32_t)((p.M + TILE - 1) / TILE), tn = (uint32_t)((p.N + TILE - 1) / TILE);
    if (blockIdx.y && workgroup_id() >= tm * tn) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, 1);
    const int64_t m0 = (int64_t)id.m * TILE, n0 = (int64_t)id.n * TILE;
    const int K = (int)p.K, steps = (K + KT - 1) / KT;

    i16v acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    // a thread's slots: the row (rows that do not exist give way to the last one)
    // and the place in a stage
    const int8_t *la[L], *lb[L];
    int at[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int e = i * NT + tid, r = S.slot_row(e);
        la[i] = p.a + (m0 + r < p.M ? m0 + r : p.M - 1) * p.lda;
        lb[i] = p.b + (n0 + r < p.N ? n0 + r : p.N - 1) * p.ldb;
        at[i] = 2 * S.slot_k(e);
    }
    raw16 ca[L], cb[L];
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int k = s * KT + at[i];
            ca[i] = K < 16 ? load16_narrow(la[i], k, K) : load16(la[i], k, K);
            cb[i] = K < 16 ? load16_narrow(lb[i], k, K) : load16(lb[i], k, K);
        }
    };
    fetch(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int k = s * KT + at[i];
            if (K >= 16) {
                settle16<int8_t>(ca[i], k, K);
                settle16<int8_t>(cb[i], k, K);
            }
            *reinterpret_cast<raw16*>(smem + (i * NT + tid) * 16) = ca[i];
            *reinterpret_cast<raw16*>(smem + S.bytes() + (i * NT + tid) * 16) = cb[i];
        }
        __syncthreads();
        if (s + 1 < steps) fetch(s + 1);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            u4 fa[MI], fb[NI];
#pragma unroll
            for (int i = 0; i < MI; ++i) fa[i] = *reinterpret_cast<const u4*>(smem + frag_byte(S, wm + 32 * i, 16 * kk, lane, 0));
#pragma unroll
            for (int j = 0; j < NI; ++j)
                fb[j] = *reinterpret_cast<const u4*>(smem + S.bytes() + frag_byte(S, wn + 32 * j, 16 * kk, lane, 0));
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mma(fb[j], fa[i], acc[i][j]);
        }
    }
    write_tile<T, MI, NI>(p, m0 + wm, n0 + wn, acc, smem, lane, wave);
}

}  // namespace

int64_t dense_int8_workspace(int64_t, int64_t, int64_t) { return 0; }

cliff_status launch_dense_int8(int dtype, const DenseInt8Args& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const Int8Args p{a.M, a.N, a.K, a.x, a.ldx, a.w, a.ldw, a.x_scale, a.w_scale,
                         a.bias, a.act, a.residual, a.ldr, a.y, a.ldy};
        const int64_t wgs = ceil_div(p.M, TILE) * ceil_div(p.N, TILE);
        if (wgs >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
        if (debug_enabled())
            fprintf(stderr, "cliffconv: int8 product %lld x %lld x %lld, staged tiles of %d, %lld workgroups\n",
                    (long long)p.M, (long long)p.N, (long long)p.K, TILE, (long long)wgs);
        hipLaunchKernelGGL(int8_tile_kernel<T>, grid_of(wgs), dim3(256), 0, stream, p);
        return launched();
    });
}

}  // namespace cliff
