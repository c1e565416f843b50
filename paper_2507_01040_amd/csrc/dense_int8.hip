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
    int splits;      // parts of the contraction, each by its own workgroups ...
    int64_t k_part;  // ... of this many values (a multiple of the stage's)
    int* partial;    // splits > 1: [splits][M][N], joined by another kernel
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

// Four neighbouring sums, of which some may not exist (have < 4).
__device__ inline i4 load4i(const int* p, int have)
{
    i4 v = {0, 0, 0, 0};
    if (have >= 4) __builtin_memcpy(&v, p, sizeof v);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) v[e] = p[e];
    return v;
}
__device__ inline void store4i(int* p, const i4& v, int have)
{
    if (have >= 4) __builtin_memcpy(p, &v, sizeof v);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) p[e] = v[e];
}

// Scales whose products are normal floats, and fit any sum: within 2^-62 and 2^62.
__device__ inline bool ordinary(float s)
{
    return (__builtin_bit_cast(uint32_t, s) >> 23) - 65u < 124u;  // (positive ones)
}

// What a group of four columns needs besides its sums, loaded early.
struct Ends {
    f4 scale, bias;
    bool ordinary;  // the scales
};
template <typename T>
__device__ inline Ends load_ends(const Int8Args& p, int64_t n)
{
    Ends e{f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}, true};
    if (n >= p.N || p.splits > 1) return e;  // (the join's)
    const int have = p.N - n < 4 ? (int)(p.N - n) : 4;
    e.scale = load4(p.b_scale + n, have);
    if (p.bias) e.bias = load4(static_cast<const T*>(p.bias) + n, have);
#pragma unroll
    for (int i = 0; i < 4; ++i) e.ordinary &= i >= have || ordinary(e.scale[i]);
    return e;
}

// The scales of rows m, m + step, ...
template <int R>
__device__ inline void row_scales(const Int8Args& p, int64_t m, int step, float (&s)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = p.a_scale[m + r * step < p.M ? m + r * step : p.M - 1];
}

// R rows of a group of four columns: rows m, m + step, ...  WHOLE: all of them exist (no
// branches then, so that waits for earlier loads need not wait for these stores).
template <typename T, int R, bool WHOLE = false>
__device__ inline void finish_rows(const Int8Args& p, int64_t m, int step, int64_t n, const i4 (&v)[R], const Ends& e,
                                   const float (&s)[R])
{
    const int have = WHOLE || p.N - n >= 4 ? 4 : (int)(p.N - n);
    f4 res[R];
    bool plain = e.ordinary;
    if (p.residual)
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (WHOLE || m + r * step < p.M)
                res[r] = load4(static_cast<const T*>(p.residual) + (m + r * step) * p.ldr + n, have);
#pragma unroll
    for (int r = 0; r < R; ++r) plain &= ordinary(s[r]);
    f4 u[R];
    if (plain) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) u[r][i] = fmaf((float)v[r][i], s[r] * e.scale[i], e.bias[i]);
    } else {
        // the scale of smaller magnitude first: neither product leaves fp32 where the result
        // does not (comparisons keep a NaN)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool less = fabsf(s[r]) < fabsf(e.scale[i]);
                u[r][i] = fmaf((float)v[r][i] * (less ? s[r] : e.scale[i]), less ? e.scale[i] : s[r], e.bias[i]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!WHOLE && m + r * step >= p.M) break;
        activate4<sizeof(T) == 4>(p.act, u[r]);
        if (p.residual) u[r] += res[r];
        store4(static_cast<T*>(p.y) + (m + r * step) * p.ldy + n, u[r], have);
    }
}

// The outputs of a wave's MI x NI blocks of 32 x 32 from row m1, column n1 on: 32
// rows at a time through LDS, so that 16 lanes hold 64 neighbouring columns of a
// row.  Begins with a barrier: the stages there are done with.
constexpr int EW = 64 + 4;  // integers per row there
template <typename T, int MI, int NI>
__device__ inline void write_tile(const Int8Args& p, const TileId& id, int64_t m1, int64_t n1,
                                  const i16v (&acc)[MI][NI], char* smem, int lane, int wave)
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
// rows at a time: as many as the registers beside the accumulators hold
            constexpr int R = MI > 1 ? 4 : 8;
#pragma unroll 1
            for (int h = 0; h < 8 / R; ++h) {
                const int r0 = 16 * h + (lane >> 4);
                const int64_t m = m1 + 32 * i + r0;
                i4 v[R];
#pragma unroll
                for (int r = 0; r < R; ++r) v[r] = *reinterpret_cast<const i4*>(tile + (r0 + 4 * r) * EW + 4 * (lane & 15));
                if (p.splits > 1) {
                    const int have = p.N - n < 4 ? (int)(p.N - n) : 4;
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (m + 4 * r < p.M) store4i(p.partial + (id.split * p.M + m + 4 * r) * p.N + n, v[r], have);
                } else {
                    float s[R];
                    row_scales(p, m, 4, s);
                    finish_rows<T, R>(p, m, 4, n, v, ends, s);
                }
            }
        }
        wave_fence();
    }
}

// BM x BN outputs per workgroup of WR x WC waves, stages of 64 contraction values in
// LDS slots of 16 (dense_geom.hpp counts them as 8 of 16 bits).  Rows that are 16-byte
// aligned and whole slots: stages go from memory straight to LDS, three ahead in a
// ring of four buffers, so that the wait for a stage is for loads that were issued
// two stages before; it stands, with the barrier, between the two groups of products
// of a stage, and the first fragments of the next stage are read under the second.
//
// Bound by the power of the matrix cores where there is much to do: 4096 x 4096 x 8192
// with GELU 149 to 158 us (1740 to 1840 TOPS), 112 with zeros for integers; 8192^3 480
// us (2290 TOPS).  64 x 64 tiles are for small ones: 1024^3 7.7 us, 10.9 with 128 x 128
// and 20.9 with 256 x 256, whose times at 4096^3 are 149, 90 and 73.
constexpr int RING = 4, KT = 64;
template <typename T, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void int8_direct_kernel(Int8Args p)
{
    constexpr int NT = 64 * WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32;
    constexpr Stage SA{BM, KT / 2, true}, SB{BN, KT / 2, true};
    constexpr int LA = SA.slots() / NT, LB = SB.slots() / NT, L = LA + LB, PA = SA.bytes(), BUF = PA + SB.bytes();
    static_assert(WN == 64 && KT == 64 && L % MI == 0, "shape");
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WC * WM, wn = wave % WC * WN;
    const uint32_t tm = (uint32_t)((p.M + BM - 1) / BM), tn = (uint32_t)((p.N + BN - 1) / BN);
    if (blockIdx.y && workgroup_id() >= tm * tn * p.splits) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, p.splits);
    const int64_t m0 = (int64_t)id.m * BM, n0 = (int64_t)id.n * BN, k0 = id.split * p.k_part;
    const int kn = (int)(p.K - k0 < p.k_part ? p.K - k0 : p.k_part), steps = (kn + KT - 1) / KT;
    const int8_t* const a = p.a + m0 * p.lda + k0;
    const int8_t* const b = p.b + n0 * p.ldb + k0;

    i16v acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    u4 fa[2][MI], fb[2][NI];
    auto read_one = [&](int set, const char* buf, int kk, int f) {  // columns' fragments first
        if (f < NI)
            fb[set][f] = *reinterpret_cast<const u4*>(buf + PA + frag_byte(SB, wn + 32 * f, 16 * kk, lane, 0));
        else
            fa[set][f - NI] = *reinterpret_cast<const u4*>(buf + frag_byte(SA, wm + 32 * (f - NI), 16 * kk, lane, 0));
    };
    // byte offsets of a thread's slots from a stage's start; rows that do not exist are
    // zeros
    uint32_t off[L];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int e = i * NT + tid, r = SA.slot_row(e);
        off[i] = m0 + r < p.M ? (uint32_t)(r * p.lda + 2 * SA.slot_k(e)) : NOWHERE;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int e = i * NT + tid, r = SB.slot_row(e);
        off[LA + i] = n0 + r < p.N ? (uint32_t)(r * p.ldb + 2 * SB.slot_k(e)) : NOWHERE;
    }
    // Load i of stage s; of stages past the last one, zeros (as many loads are under way
    // in every step).
    auto load = [&](int s, int i) {
        const int l = i < LA ? i : i - LA, left = kn - s * KT;
        const Stage& S = i < LA ? SA : SB;
        const uint32_t o = left < KT && 2 * S.slot_k(l * NT + tid) >= left ? NOWHERE : off[i];
        load_to_lds((i < LA ? a : b) + (int64_t)s * KT, o,
                    smem + s % RING * BUF + (i < LA ? 0 : PA) + wave * 1024 + l * NT * 16);
    };
    // Products of a group of 32 values, with the reads of the next one's fragments
    // (next: its buffer).  The output's columns are the matrix instruction's rows: a
    // lane's groups of four sums are neighbours.
    auto group = [&](int set, const char* next, int kk, auto loads) {
        constexpr int F = MI + NI;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int f = i * F / MI; f < (i + 1) * F / MI; ++f) read_one(set ^ 1, next, kk, f);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mma(fb[set][j], fa[set][i], acc[i][j]);
#pragma unroll
            for (int l = i * L / MI; l < (i + 1) * L / MI; ++l) loads(l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int s = 0; s < RING - 1; ++s)
#pragma unroll
        for (int i = 0; i < L; ++i) load(s, i);
    wait_direct_but<2 * L>();
    __syncthreads();
#pragma unroll
    for (int f = 0; f < MI + NI; ++f) read_one(0, smem, 0, f);
    for (int s = 0; s < steps; ++s) {
        group(0, smem + s % RING * BUF, 1, [](int) {});
        wait_direct_but<L>();
        // Every wave has the fragments of stage s - 1, whose buffer the loads now take:
        // its products with them stand before the barrier.
        barrier_alone();
        __builtin_amdgcn_sched_barrier(0);
        // (the last step reads what no product uses)
        group(1, smem + (s + 1) % RING * BUF, 0, [&](int i) { load(s + RING - 1, i); });
    }
    wait_direct();
    write_tile<T, MI, NI>(p, id, m0 + wm, n0 + wn, acc, smem, lane, wave);
}

// The same for rows of any alignment and width: stages of 128 values, whose slots go
// through registers, one stage ahead.  Bound by the latency of a stage: 1003 x 777 x 1531
// with GELU and residual 18 us in tiles of 64, 29 in tiles of 128, whose 96 workgroups
// leave the epilogue to few waves.
constexpr int KT_STAGED = 128;
template <typename T, int TILE, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void int8_staged_kernel(Int8Args p)
{
    constexpr int KT = KT_STAGED, NT = 64 * WR * WC, WM = TILE / WR, WN = TILE / WC, MI = WM / 32, NI = WN / 32;
    constexpr Stage S{TILE, KT / 2, true};
    constexpr int L = S.slots() / NT, KK = KT / 32, EPILOGUE = WR * WC * 32 * EW * 4;
    static_assert(WN == 64, "shape");
    __shared__ __align__(16) char smem[2 * S.bytes() > EPILOGUE ? 2 * S.bytes() : EPILOGUE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WC * WM, wn = wave % WC * WN;
    const uint32_t tm = (uint32_t)((p.M + TILE - 1) / TILE), tn = (uint32_t)((p.N + TILE - 1) / TILE);
    if (blockIdx.y && workgroup_id() >= tm * tn * p.splits) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, p.splits);
    const int64_t m0 = (int64_t)id.m * TILE, n0 = (int64_t)id.n * TILE;
    const int K = (int)p.K, k0 = (int)(id.split * p.k_part), k1 = K - k0 < p.k_part ? K : k0 + (int)p.k_part;
    const int steps = (k1 - k0 + KT - 1) / KT;

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
    // (a part that is not the last one ends with a whole stage: pieces past its end are
    // past the row's)
    raw16 ca[L], cb[L];
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int k = k0 + s * KT + at[i];
            ca[i] = K < 16 ? load16_narrow(la[i], k, K) : load16(la[i], k, K);
            cb[i] = K < 16 ? load16_narrow(lb[i], k, K) : load16(lb[i], k, K);
        }
    };
    fetch(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        const bool whole = k0 + (s + 1) * KT <= K;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (!whole && K >= 16) {
                settle16<int8_t>(ca[i], k0 + s * KT + at[i], K);
                settle16<int8_t>(cb[i], k0 + s * KT + at[i], K);
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
    write_tile<T, MI, NI>(p, id, m0 + wm, n0 + wn, acc, smem, lane, wave);
}

// Joins the parts of a split contraction and finishes the outputs: a thread for each
// group of four columns, bound by the read of the parts.
template <typename T>
__global__ __launch_bounds__(256) void int8_join_kernel(Int8Args p)
{
    const int64_t nq = (p.N + 3) / 4, plane = p.M * p.N, i = workgroup_id() * 256ll + threadIdx.x;
    const int64_t m = i >> 32 ? i / nq : (int64_t)((uint32_t)i / (uint32_t)nq), n = (i - m * nq) * 4;
    if (m >= p.M) return;
    const int have = p.N - n < 4 ? (int)(p.N - n) : 4, splits = p.splits;
    Int8Args whole = p;
    whole.splits = 1;
    const Ends ends = load_ends<T>(whole, n);
    const int* const q = p.partial + m * p.N + n;
    i4 v[1] = {i4{0, 0, 0, 0}};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v[0] += load4i(q + s * plane, have);
    const float s[1] = {p.a_scale[m]};
    finish_rows<T, 1>(p, m, 1, n, v, ends, s);
}

// Few rows (16 MB at most): bound by the read of the weight.  A workgroup streams 16
// of its outputs' rows once, its eight waves an eighth of the contraction each, D
// stages of 128 values ahead, and they join their sums in LDS; as for 16-bit types
// (rows.hpp), with matrix instructions of 16 x 16 outputs and 64 values.  1 x 4096 x 8192
// 10.5 us, 24 x 8192 x 4096 8.8; in tiles 38 and 75.
template <typename T, int MB>
__global__ __launch_bounds__(512, 2) void int8_rows_kernel(Int8Args p)
{
    constexpr int D = MB == 4 ? 3 : MB == 1 ? 8 : 4;  // what the registers hold
    constexpr int W = 16 + 4, OWN = (MB + 1) * LINES, PLANE = MB * 16 * W;
    __shared__ __align__(16) char smem[8 * (PLANE * 4 > OWN ? PLANE * 4 : OWN)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowsPart<128> part(p.N, p.K, 16, wave);
    const int8_t* const b = p.b + part.n0 * p.ldb;
    i4 acc[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i] = i4{0, 0, 0, 0};
    struct St {
        raw16 x[MB][2], w[2];
    };
    char* const own = smem + wave * OWN;
    Lines al[MB], bl(0, part.cols, p.ldb, lane, int8_t{});
#pragma unroll
    for (int i = 0; i < MB; ++i) al[i] = Lines(16 * i, p.M, p.lda, lane, int8_t{});
    auto load = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) al[i].load(f.x[i], p.a + k);
        bl.load(f.w, b + k);
    };
    auto load_last = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::load_last(f.x[i], p.a, 16 * i, p.M, p.lda, k, part.k1, lane);
        Lines::load_last(f.w, b, 0, part.cols, p.ldb, k, part.k1, lane);
    };
    auto use = [&](St& f) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::write(f.x[i], own + i * LINES, lane);
        Lines::write(f.w, own + MB * LINES, lane);
        wave_fence();
        raw16 w[2], x[MB][2];
        Lines::read(w, own + MB * LINES, lane);
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::read(x[i], own + i * LINES, lane);
        wave_fence();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < MB; ++i)
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, w[j]), __builtin_bit_cast(i4, x[i][j]),
                                                               acc[i], 0, 0, 0);
    };
    part.template run<D, St>(load, load_last, use);

    int* const lds = reinterpret_cast<int*>(smem);
    const int r = threadIdx.x / 4, c = 4 * (threadIdx.x % 4);
    const int64_t n = part.n0 + c;
    const Ends ends = load_ends<T>(p, n);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i)
        *reinterpret_cast<i4*>(lds + wave * PLANE + (16 * i + (lane & 15)) * W + 4 * (lane >> 4)) = acc[i];
    __syncthreads();
    if (r >= 16 * MB || r >= p.M || n >= p.N) return;
    i4 v[1] = {i4{0, 0, 0, 0}};
#pragma unroll
    for (int w = 0; w < 8; ++w) v[0] += *reinterpret_cast<const i4*>(lds + w * PLANE + r * W + c);
    const float s[1] = {p.a_scale[r]};
    finish_rows<T, 1>(p, r, 1, n, v, ends, s);
}

// Many rows and a short contraction: bound by the write of y (and its activation), and
// a tile has too few stages to hide its begin and end.  So 128 outputs' weights stay in
// LDS (a panel), and each of four waves streams blocks of 32 rows past it without
// barriers, x from memory straight into fragments that stay for all columns, the next
// block's loads under the work on this one.  The panel lies as [slot][column] in 16-byte slots, slot 2 kk + h
// with the 16 values of half-wave h in product group kk, read without bank conflicts.
// 131072 x 128 x 512 fp32 60 us (4.6 TB/s, in tiles 76), with GELU 90; 65536 x 128 x 512
// bf16 23 us (tiles 33).  Four waves, so that three workgroups' registers fit a compute
// unit: eight with 128 registers spilled, 32 us.
constexpr int PANEL = 128, PANEL_EW = 32 + 4;
constexpr int PANEL_WAVES = 4;
template <typename T, int KK>
__global__ __launch_bounds__(64 * PANEL_WAVES, 3) void int8_panel_kernel(Int8Args p)
{
    constexpr int SLOTS = 2 * KK * PANEL;
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    float* const scales = reinterpret_cast<float*>(smem + SLOTS * 16);
    float* const bias = scales + PANEL;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int* const tile = reinterpret_cast<int*>(bias + PANEL) + wave * 32 * PANEL_EW;
    const uint32_t panels = (uint32_t)((p.N + PANEL - 1) / PANEL), t = xcd_run(blockIdx.x, gridDim.x);
    const int64_t n0 = (int64_t)(t % panels) * PANEL, stride = (int64_t)(gridDim.x / panels) * PANEL_WAVES;
    const int K = (int)p.K;
    if (tid < PANEL) {
        scales[tid] = n0 + tid < p.N ? p.b_scale[n0 + tid] : 1.f;
        bias[tid] = p.bias && n0 + tid < p.N ? (float)static_cast<const T*>(p.bias)[n0 + tid] : 0.f;
    }
    for (int i = tid; i < SLOTS; i += 64 * PANEL_WAVES) {
        const int64_t n = n0 + i % PANEL < p.N ? n0 + i % PANEL : p.N - 1;  // (columns that do not exist are not written)
        raw16 v = load16(p.b + n * p.ldb, i / PANEL * 16, K);
        settle16<int8_t>(v, i / PANEL * 16, K);
        *reinterpret_cast<raw16*>(smem + i * 16) = v;
    }
    __syncthreads();

    const int64_t blocks = (p.M + 31) / 32, b0 = (int64_t)(t / panels) * PANEL_WAVES + wave;
    if (b0 >= blocks) return;
    raw16 x[KK], next[KK];
    float s[4], next_s[4];
    // A block's rows (those that do not exist give way to the last one) and their scales.
    auto load = [&](int64_t blk) {
        const int64_t row = 32 * blk + (lane & 31);
        const int8_t* const line = p.a + (row < p.M ? row : p.M - 1) * p.lda;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) next[kk] = load16(line, 32 * kk + 16 * half, K);
        row_scales(p, 32 * blk + (lane >> 3), 8, next_s);
    };
    const char* const mine = smem + (half * PANEL + (lane & 31)) * 16;
    load(b0);
    for (int64_t blk = b0; blk < blocks; blk += stride) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            x[kk] = next[kk];
            if (K < 32 * KK) settle16<int8_t>(x[kk], 32 * kk + 16 * half, K);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = next_s[r];
        if (blk + stride < blocks) load(blk + stride);
        // 32 columns at a time through LDS: 8 lanes hold a row's.
        const int64_t m = 32 * blk + (lane >> 3);
        const bool whole = 32 * blk + 32 <= p.M && n0 + PANEL <= p.N;
        auto finish = [&](const i16v& c, int j) {
            wave_fence();
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<i4*>(tile + (lane & 31) * PANEL_EW + 8 * g + 4 * half) =
                    i4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
            wave_fence();
            i4 v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = *reinterpret_cast<const i4*>(tile + ((lane >> 3) + 8 * r) * PANEL_EW + 4 * (lane & 7));
            const int c0 = 32 * j + 4 * (lane & 7);
            Ends e{*reinterpret_cast<const f4*>(scales + c0), *reinterpret_cast<const f4*>(bias + c0), true};
#pragma unroll
            for (int i = 0; i < 4; ++i) e.ordinary &= ordinary(e.scale[i]);
            if (whole) finish_rows<T, 4, true>(p, m, 8, n0 + c0, v, e, s);
            else if (n0 + c0 < p.N) finish_rows<T, 4>(p, m, 8, n0 + c0, v, e, s);
        };
#pragma unroll 1
        for (int j = 0; j < PANEL / 32; ++j) {
            i16v acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                acc = mma(*reinterpret_cast<const u4*>(mine + (2 * kk * PANEL + 32 * j) * 16), __builtin_bit_cast(u4, x[kk]), acc);
            finish(acc, j);
        }
    }
}

// How a product is cut: square tiles, and parts of the contraction, by the times in ns
// of 128 values with one workgroup on each compute unit and with as many as fit, and
// of a workgroup's begin and end.
struct Cut {
    int tile, splits;
    int64_t k_part;
    double ns;  // what it is expected to take
};
struct TileTimes {
    int tile, fit;
    double alone, full, ends;
};
// Fitted to measured times (MI355X; 44 products of 65 to 65536 rows with 1 to 32 parts
// each, aligned and not; 15 % off on average; the cuts that they choose take 1.4 %
// longer than the best ones, 16 % at worst).
constexpr TileTimes T_DIRECT[] = {{256, 1, 990, 990, 11000}, {128, 3, 360, 1460, 8300}, {64, 2, 270, 410, 3200}},
                    T_STAGED[] = {{128, 2, 740, 740, 10500}, {64, 2, 960, 1000, 1800}};

Cut cut(int64_t M, int64_t N, int64_t K, bool direct)
{
    const int64_t cus = std::max(device_cus(), 1), steps = ceil_div(K, 128);
    Cut best{0, 1, 0, 0};
    const auto weigh = [&](const TileTimes& t) {
        const int64_t tiles = ceil_div(M, t.tile) * ceil_div(N, t.tile);
        for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (want > steps) break;
            const int64_t per = ceil_div(steps, want), splits = ceil_div(steps, per);
            const int64_t wgs = tiles * splits, rounds = wgs / (cus * t.fit), rest = wgs % (cus * t.fit);
            double ns = rounds * (per * t.full + t.ends);
            if (rest) ns += per * (rest <= cus ? t.alone : t.full) + t.ends;
            // the join: a launch, and the partial sums written and read
            if (splits > 1) ns += 2800 + (double)M * N * 4 * 2 * splits / 7400;
            if (best.ns == 0 || ns < best.ns) best = Cut{t.tile, (int)splits, per * 128, ns};
        }
    };
    if (direct)
        for (const TileTimes& t : T_DIRECT) weigh(t);
    else
        for (const TileTimes& t : T_STAGED) weigh(t);
    return best;
}

// What the kernel of few rows is for: rows, row strides (32-bit offsets), and outputs
// (2^32 threads of a grid).
constexpr int64_t FEW_ROWS = 64, FEW_LD = 1 << 24, FEW_N = 1 << 26;

// Its time in ns, from the bytes that a compute unit takes in: every workgroup reads
// all of x.
double few_rows_ns(int64_t M, int64_t N, int64_t K)
{
    const int rows = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    const double rounds = std::max(1., (double)ceil_div(N, 16) / std::max(device_cus(), 1));
    return 3500 + rounds * (double)(K * (rows + 16)) / 75;
}

// The longest contraction of the panel kernel, and rows and outputs from which it is level
// with the tiles or ahead (us, panels and tiles, bf16, K 128: 2048 x 2048 outputs 7.2 and
// 7.5, 4096 x 512 6.6 and 6.5, 16384 x 128 6.7 and 7.3, 65536 x 512 22.4 and 32.9; 8192 x
// 128 6.4 and 5.6; 20000 x 1000 with K 256, which would fit too, 30.9 and 26.4).
constexpr int64_t PANEL_K = 128, PANEL_ROWS = 2048, PANEL_OUTPUTS = 1 << 21;

bool aligned_rows(const void* x, int64_t ld, int64_t width)
{
    return ((uintptr_t)x & 15) == 0 && ld % 16 == 0 && width % 16 == 0 && ld <= (1 << 22);
}

template <typename T>
cliff_status int8_product(Int8Args p, hipStream_t stream)
{
    const bool direct = aligned_rows(p.a, p.lda, p.K) && aligned_rows(p.b, p.ldb, p.K);
    const Cut c = cut(p.M, p.N, p.K, direct);
    p.splits = 1;
    const auto say = [&](const char* name, int64_t wgs) {
        if (debug_enabled())
            fprintf(stderr, "cliffconv: int8 product %lld x %lld x %lld, %s, %lld workgroups, %d splits\n", (long long)p.M,
                    (long long)p.N, (long long)p.K, name, (long long)wgs, p.splits);
    };
    if (p.M <= FEW_ROWS && p.K >= 16 && p.lda <= FEW_LD && p.ldb <= FEW_LD && p.N <= FEW_N &&
        few_rows_ns(p.M, p.N, p.K) < c.ns) {
        const int64_t wgs = ceil_div(p.N, 16);
        say("few rows", wgs);
        const auto go = [&](auto k) { hipLaunchKernelGGL(k, dim3((unsigned)wgs), dim3(512), 0, stream, p); };
        if (p.M <= 16) go(int8_rows_kernel<T, 1>);
        else if (p.M <= 32) go(int8_rows_kernel<T, 2>);
        else go(int8_rows_kernel<T, 4>);
        return launched();
    }
    const int64_t panels = ceil_div(p.N, PANEL);
    if (p.M >= PANEL_ROWS && p.M * p.N >= PANEL_OUTPUTS && p.K <= PANEL_K && p.K >= 16 && panels < 1 << 22) {
        const int64_t cus = std::max(device_cus(), 1);
        const int64_t wgs = panels * std::min(std::max<int64_t>(1, 3 * cus / panels), ceil_div(p.M, 32 * PANEL_WAVES));
        say("panels", wgs);
        const auto go = [&](auto k, int KK) {
            const int lds = 2 * KK * PANEL * 16 + (2 * PANEL + PANEL_WAVES * 32 * PANEL_EW) * 4;
            hipLaunchKernelGGL(k, dim3((unsigned)wgs), dim3(64 * PANEL_WAVES), lds, stream, p);
        };
        if (p.K <= 64) go(int8_panel_kernel<T, 2>, 2);
        else go(int8_panel_kernel<T, 4>, 4);
        return launched();
    }
    p.splits = c.splits;
    p.k_part = c.k_part;
    const int64_t wgs = ceil_div(p.M, c.tile) * ceil_div(p.N, c.tile) * p.splits;
    if (wgs >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    char name[40];
    snprintf(name, sizeof name, "%s tiles of %d", direct ? "direct" : "staged", c.tile);
    say(name, wgs);
    // LDS: the ring of stages, or what write_tile takes
    const auto go = [&](auto k, int threads, int lds) { hipLaunchKernelGGL(k, grid_of(wgs), dim3(threads), lds, stream, p); };
    if (direct && c.tile == 256) go(int8_direct_kernel<T, 256, 256, 2, 4>, 512, RING * 2 * 256 * KT);
    else if (direct && c.tile == 128) go(int8_direct_kernel<T, 128, 128, 2, 2>, 256, RING * 2 * 128 * KT);
    else if (direct) go(int8_direct_kernel<T, 64, 64, 2, 1>, 128, RING * 2 * 64 * KT);
    else if (c.tile == 128) go(int8_staged_kernel<T, 128, 2, 2>, 256, 0);
    else go(int8_staged_kernel<T, 64, 2, 1>, 128, 0);
    const cliff_status s = launched();
    if (s != CLIFF_OK || p.splits == 1) return s;
    const int64_t blocks = ceil_div(p.M * ceil_div(p.N, 4), 256);
    if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    hipLaunchKernelGGL(int8_join_kernel<T>, grid_of(blocks), dim3(256), 0, stream, p);
    return launched();
}

}  // namespace

int64_t dense_int8_workspace(int64_t M, int64_t K, int64_t N)
{
    int64_t n = 0;
    for (const bool direct : {false, true}) {
        const Cut c = cut(M, N, K, direct);
        if (c.splits > 1) n = std::max(n, c.splits * M * N * 4);
    }
    return ceil_div(n, 256) * 256;
}

cliff_status launch_dense_int8(int dtype, const DenseInt8Args& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return int8_product<T>(Int8Args{a.M, a.N, a.K, a.x, a.ldx, a.w, a.ldw, 1, 0, static_cast<int*>(a.workspace),
                                        a.x_scale, a.w_scale, a.bias, a.act, a.residual, a.ldr, a.y, a.ldy},
                               stream);
    });
}

}  // namespace cliff
