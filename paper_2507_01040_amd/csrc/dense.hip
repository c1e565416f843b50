// Dense layer with its epilogue, and its gradient: three matrix products
//   y = x w,  dx = g w^T,  dw = x^T g
// of one kernel, which takes either operand contiguous along the contraction or
// along the output (Stage::KM).
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include "dense_geom.hpp"
#include "ff_common.hpp"
#include "lds_load.hpp"
#include "rows.hpp"
#include "split.hpp"

namespace cliff {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// C[m, n] = scale sum_k A(m, k) B(n, k): operand X is [R, K] with row stride ld
// (KM) or [K, R] with it.
struct ProductArgs {
    int64_t M, N, K;
    const void* a;
    int64_t lda;
    const void* b;
    int64_t ldb;
    int splits;       // parts of the contraction, each by its own workgroups ...
    float scale;
    int64_t k_part;   // ... of this many values (a multiple of the stage's)
    float* partial;   // splits > 1: fp32 [splits][M][N], joined by another kernel
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

// Eight elements in 16-byte pieces (load16): one of a 16-bit type, two of fp32.
template <typename T>
struct Chunk {
    raw16 v[sizeof(T) / 2];
};

// The three bf16 parts of eight floats.
__device__ inline void split_chunk(const Chunk<float>& c, u4 (&t)[3])
{
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const f4 v = __builtin_bit_cast(f4, c.v[h >> 1]);
        const Parts q = split2(v[2 * (h & 1)], v[2 * (h & 1) + 1]);
#pragma unroll
        for (int u = 0; u < 3; ++u) t[u][h] = q.t[u];
    }
}

template <typename T>
__device__ inline f16v mma(const u4& x, const u4& y, const f16v& c)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, x), __builtin_bit_cast(h8, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, x), __builtin_bit_cast(b8, y), c, 0, 0, 0);
}

// A Stage as a type, so that its shape is known when a function is compiled.
template <int R_, int KT_, bool KM_>
struct StageOf {
    static constexpr Stage s{R_, KT_, KM_};
    static constexpr bool KM = KM_;
};

// Stages of one operand's tile, from its first row and contraction value.
template <typename T, typename SO, int NT>
struct Operand {
    static constexpr Stage S = SO::s;
    static constexpr int L = S.slots() / NT;  // slots per thread
    static_assert(S.slots() % NT == 0, "whole slots");
    const T* x;
    int64_t ld;
    int rows;      // of the tile that exist
    int64_t vals;  // contraction values that exist
    int64_t width;  // elements of a line of memory before the tile's end

    // Byte offsets of a thread's slots from a stage's start (direct loads).
    __device__ void offsets(uint32_t (&off)[L], int tid) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = i * NT + tid, r = S.slot_row(e), k = S.slot_k(e);
            off[i] = r < rows ? (uint32_t)((S.KM ? r * ld + k : k * ld + r) * 2) : NOWHERE;
        }
    }
    // Piece i of L of stage s straight to LDS; slots past the last value become
    // zeros.  The caller waits (wait_direct) before the barrier that makes the
    // stage readable.
    __device__ void direct(uint32_t off, int i, int s, char* to, int tid, int wave) const
    {
        const int n = left(s);
        if (n < S.KT && S.slot_k(i * NT + tid) >= n) off = NOWHERE;
        load_to_lds(x + (S.KM ? (int64_t)s * S.KT : (int64_t)s * S.KT * ld), off, to + wave * 1024 + i * NT * 16);
    }
    __device__ int left(int s) const  // of a stage's values, those that exist
    {
        const int64_t n = vals - (int64_t)s * S.KT;
        return n < S.KT ? (int)n : S.KT;
    }
    // Loads through registers.  Whether the rows are whole slots: those that do
    // not exist then give way to others, for nothing reads their products.
    __device__ bool plain() const { return S.KM || rows == S.R || rows % 8 == 0; }
    // A thread's slots of the first stage of a plain tile; the next stage's are
    // `advance` elements on.
    __device__ void pointers(const T* (&at)[L], int tid) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = i * NT + tid, r = S.slot_row(e), k = S.slot_k(e), last = S.KM ? rows - 1 : rows - 8;
            at[i] = x + (S.KM ? (r < last ? r : last) * ld + k : k * ld + (r < last || last < 0 ? r : last));
        }
    }
    __device__ int64_t advance() const { return S.KM ? S.KT : S.KT * ld; }
    // A stage into registers ...
    __device__ void fetch_whole(Chunk<T> (&c)[L], const T* (&at)[L]) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            __builtin_memcpy(&c[i], at[i], sizeof c[i]);
            at[i] += advance();
        }
    }
    // (of a tile that is not plain or a stage that is not whole; what it lacks is
    // zeroed in store)
    __device__ void fetch(Chunk<T> (&c)[L], const T* (&at)[L], int s, int tid) const
    {
        const int n = left(s);
        if (n == S.KT && plain()) return fetch_whole(c, at);
        const T* const stage = x + s * advance();
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = i * NT + tid, r = S.slot_row(e), k = S.slot_k(e);
            // the slot's line, from the tile's first element there; lines that do
            // not exist give way to the last one
            const int line = S.KM ? r : k, lines = S.KM ? rows : n, pos = S.KM ? k : r, end = S.KM ? n : rows;
            const T* const p = stage + (line < lines ? line : lines - 1) * ld;
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h)
                c[i].v[h] = width < per16<T> ? load16_narrow(p, pos + h * per16<T>, end)
                                             : load16(p, pos + h * per16<T>, end);
            at[i] += advance();
        }
    }
    // ... and from there to LDS, fp32 as three planes.
    static __device__ void put(const Chunk<T> (&c)[L], char* to, int tid)
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            char* const at = to + (i * NT + tid) * 16;
            if constexpr (sizeof(T) == 4) {
                u4 t[3];
                split_chunk(c[i], t);
#pragma unroll
                for (int u = 0; u < 3; ++u) *reinterpret_cast<u4*>(at + u * S.bytes()) = t[u];
            } else {
                *reinterpret_cast<u4*>(at) = c[i].v[0];
            }
        }
    }
    __device__ void store(Chunk<T> (&c)[L], int s, char* to, int tid) const
    {
        const int n = left(s);
        if (n < S.KT || !plain())
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int e = i * NT + tid, r = S.slot_row(e), k = S.slot_k(e);
#pragma unroll
                for (int h = 0; h < (int)sizeof(T) / 2; ++h)
                    if (!S.KM && k >= n) c[i].v[h] = raw16{0, 0, 0, 0};
                    else if (width >= per16<T>) settle16<T>(c[i].v[h], (S.KM ? k : r) + h * per16<T>, S.KM ? n : rows);
            }
        put(c, to, tid);
    }
    // The fragment of rows row0 to + 31 and values k to + 15 of a stage in LDS.
    static __device__ u4 frag(const char* from, int row0, int k, int lane)
    {
        if constexpr (SO::KM) {
            return *reinterpret_cast<const u4*>(from + frag_byte(S, row0, k, lane, 0));
        } else {
            typedef __attribute__((address_space(3))) s4 ls4;
            struct {
                s4 x, y;
            } z{__builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4*)(from + frag_byte(S, row0, k, lane, 0))),
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4*)(from + frag_byte(S, row0, k, lane, 1)))};
            return __builtin_bit_cast(u4, z);
        }
    }
    // element (r, k), zero outside
    __device__ float at(int r, int64_t k) const
    {
        return r < rows && k < vals ? (float)x[S.KM ? r * ld + k : k * ld + r] : 0.f;
    }
};

// What the epilogue of a group of four columns needs besides their sums, loaded
// early.
struct Ends {
    f4 bias;
    uint64_t key;
    uint32_t step;
};
template <typename T>
__device__ inline Ends load_ends(const ProductArgs& p, int64_t n)
{
    Ends e{f4{0.f, 0.f, 0.f, 0.f}, 0, 0};
    if (p.splits > 1) return e;  // the join's
    if (p.bias && n < p.N) e.bias = load4(static_cast<const T*>(p.bias) + n, p.N - n < 4 ? (int)(p.N - n) : 4);
    if (p.drop.rng) {
        e.key = (uint64_t)p.drop.rng[0];
        e.step = (uint32_t)p.drop.rng[1];
    }
    return e;
}

// R rows of a group of four columns: rows m, m + step, ...  WHOLE: all of them
// exist (no branches then, so that waits for earlier loads need not wait for
// these stores).
template <typename T, int R, bool WHOLE = false>
__device__ inline void finish_rows(const ProductArgs& p, int64_t m, int step, int64_t n, const f4 (&v)[R],
                                   const Ends& e)
{
    const int have = WHOLE || p.N - n >= 4 ? 4 : (int)(p.N - n);
    f4 res[R];
    if (p.residual) {
        const T* const from = static_cast<const T*>(p.residual) + m * p.ldr + n;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (WHOLE || m + r * step < p.M) res[r] = load4(from + r * (step * p.ldr), have);
    }
    T* const y = static_cast<T*>(p.y) + m * p.ldy + n;
    T* const pre = static_cast<T*>(p.pre) + m * p.ldp + n;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!WHOLE && m + r * step >= p.M) break;
        f4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = fmaf(v[r][i], p.scale, e.bias[i]);
        if (p.pre) store4(pre + r * (step * p.ldp), u, have);
        activate4<sizeof(T) == 4>(p.act, u);
        if (p.drop.rng) drop4(p.drop, e.key, e.step, m + r * step, n, u);
        if (p.residual) u += res[r];
        store4(y + r * (step * p.ldy), u, have);
    }
}

// The outputs of a wave's MI x NI blocks of 32 x 32 from row m1, column n1 on: 32
// rows at a time through LDS, so that 16 lanes hold 64 neighbouring columns of a
// row.  Begins with a barrier: the stages there are done with.
template <typename T, int MI, int NI>
__device__ inline void write_tile(const ProductArgs& p, const TileId& id, int64_t m1, int64_t n1,
                                  const f16v (&acc)[MI][NI], char* smem, int lane, int wave)
{
    const int64_t n = n1 + 4 * (lane & 15);
    const Ends ends = load_ends<T>(p, n);
    __syncthreads();
    constexpr int EW = 64 + 4;  // floats per row there
    float* const tile = reinterpret_cast<float*>(smem) + wave * 32 * EW;
    auto put = [&](const f16v& c, int j) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f4*>(tile + (lane & 31) * EW + 32 * j + 8 * g + 4 * (lane >> 5)) =
                f4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
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
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (n < p.N) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int r0 = 16 * h + (lane >> 4);
                const int64_t m = m1 + 32 * i + r0;
                f4 v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const f4*>(tile + (r0 + 4 * r) * EW + 4 * (lane & 15));
                if (p.splits > 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (m + 4 * r < p.M)
                            store4(p.partial + (id.split * p.M + m + 4 * r) * p.N + n, v[r],
                                   p.N - n < 4 ? (int)(p.N - n) : 4);
                } else {
                    finish_rows<T, 4>(p, m, 4, n, v, ends);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// BM x BN outputs per workgroup of WR x WC waves; a stage is KT contraction
// values of 16 bits.  DIRECT: operands whose rows are 16-byte aligned and whole
// slots go from memory straight to LDS, one stage ahead in the other of two
// buffers.  Otherwise slots go through registers, one stage ahead (two ahead cost
// the second workgroup of a compute unit: 4000 x 4001 x 4096 in 275 us, not 182).
//
// Bound by the matrix cores and LDS together: a 32 x 32 x 16 product takes 32
// cycles of one of four SIMDs, a fragment 8 cycles of LDS (1 KB at 128 bytes a
// cycle).  For 16 contraction values a tile of 256 x 256 has 64 products (512
// cycles), 48 fragment reads and 16 KB of writes (512 cycles); one of 128 x 128 has
// 16 products (128 cycles) and 192 cycles of LDS.  So tiles are large where there
// are enough of them: 4000 x 4008 x 4096 bf16 112 us, 144 with 128 x 128; 1008 x 784
// x 1536, one round either way, 24.4 and 13.4.  8192^3 bf16 1290 to 1336 TFLOP/s;
// 4096 x 4096 x 8192 with GELU, dropout and both outputs 250 us, 1100 TFLOP/s.
template <typename T, bool AKM, bool BKM, int BM, int BN, int WR, int WC, int KT, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(ProductArgs p)
{
    constexpr int NT = 64 * WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32;
    static_assert(sizeof(T) == 2 && WN % 64 == 0, "shape");
    using A = Operand<T, StageOf<BM, KT, AKM>, NT>;
    using B = Operand<T, StageOf<BN, KT, BKM>, NT>;
    constexpr int PA = A::S.bytes(), BUF = PA + B::S.bytes(), KK = KT / 16;
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WC * WM, wn = wave % WC * WN;

    const uint32_t tm = (uint32_t)((p.M + BM - 1) / BM), tn = (uint32_t)((p.N + BN - 1) / BN);
    if (blockIdx.y && workgroup_id() >= tm * tn * p.splits) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, p.splits);
    const int64_t m0 = (int64_t)id.m * BM, n0 = (int64_t)id.n * BN, k0 = id.split * p.k_part;
    const int64_t kn = p.K - k0 < p.k_part ? p.K - k0 : p.k_part;
    const int steps = kn > 0 ? (int)((kn + KT - 1) / KT) : 0;
    const A a{static_cast<const T*>(p.a) + (AKM ? m0 * p.lda + k0 : k0 * p.lda + m0), p.lda,
              (int)(p.M - m0 < BM ? p.M - m0 : BM), kn, AKM ? k0 + kn : p.M};
    const B b{static_cast<const T*>(p.b) + (BKM ? n0 * p.ldb + k0 : k0 * p.ldb + n0), p.ldb,
              (int)(p.N - n0 < BN ? p.N - n0 : BN), kn, BKM ? k0 + kn : p.N};

    f16v acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    u4 fa[2][MI], fb[2][NI];
    auto read_one = [&](int set, const char* buf, int kk, int f) {  // columns' fragments first
        if (f < NI) fb[set][f] = B::frag(buf + PA, wn + 32 * f, 16 * kk, lane);
        else fa[set][f - NI] = A::frag(buf, wm + 32 * (f - NI), 16 * kk, lane);
    };
    auto read = [&](int set, const char* buf, int kk) {
#pragma unroll
        for (int f = 0; f < MI + NI; ++f) read_one(set, buf, kk, f);
    };
    // The output's columns are the matrix instruction's rows: a lane's groups of
    // four accumulators are neighbours in memory.
    auto multiply_row = [&](int set, int i) {
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mma<T>(fb[set][j], fa[set][i], acc[i][j]);
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int i = 0; i < MI; ++i) multiply_row(set, i);
    };

    if constexpr (DIRECT) {
        // The wait for a stage and the barrier stand before the last group of
        // products of the one before it, when that one's fragments have all been
        // read: the first fragments of the new stage come while those products run.
        // The loads of a stage are spread over the products of two groups (all at
        // once they keep the waves from their products for a third of the step).
        static_assert(KK % 2 == 0 && A::L == B::L && A::L % MI == 0, "groups");
        uint32_t offa[A::L], offb[B::L];
        a.offsets(offa, tid);
        b.offsets(offb, tid);
        auto load_a = [&](int s, int i) { a.direct(offa[i], i, s, smem + (s & 1) * BUF, tid, wave); };
        auto load_b = [&](int s, int i) { b.direct(offb[i], i, s, smem + (s & 1) * BUF + PA, tid, wave); };
        // Products of a group of 16 values, with the reads of the next one's
        // fragments (next: its buffer) and half of the loads of a stage.
        auto group = [&](int set, const char* next, int kk, auto loads) {
            constexpr int F = MI + NI;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
#pragma unroll
                for (int f = i * F / MI; f < (i + 1) * F / MI; ++f)
                    read_one(set ^ 1, next, kk, f);
                multiply_row(set, i);
#pragma unroll
                for (int l = i * A::L / MI; l < (i + 1) * A::L / MI; ++l) loads(l);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto nothing = [](int) {};
        if (steps > 0) {
#pragma unroll
            for (int i = 0; i < A::L; ++i) load_a(0, i);
#pragma unroll
            for (int i = 0; i < B::L; ++i) load_b(0, i);
            wait_direct();
            __syncthreads();
            if (steps > 1)
#pragma unroll
                for (int i = 0; i < A::L; ++i) load_a(1, i);
            read(0, smem, 0);
        }
        // Step s; whether there are one and two more.
        auto step = [&](int s, auto one, auto two) {
            const char* const buf = smem + (s & 1) * BUF;
            group(0, buf, 1, [&](int i) {
                if constexpr (one) load_b(s + 1, i);
            });
#pragma unroll
            for (int kk = 1; kk + 1 < KK; ++kk) group(kk & 1, buf, kk + 1, nothing);
            wait_direct();
            __syncthreads();
            // (the last step reads what no product uses)
            group(1, smem + ((s + 1) & 1) * BUF, 0, [&](int i) {
                if constexpr (two) load_a(s + 2, i);
            });
        };
        constexpr std::true_type yes;
        constexpr std::false_type no;
        int s = 0;
        for (; s + 2 < steps; ++s) step(s, yes, yes);
        if (s + 1 < steps) step(s++, yes, no);
        if (s < steps) step(s, no, no);
    } else {
        // Two fragment reads before each product, while there are any.
        auto interleave = [&](bool reads) {
            constexpr int RD = MI * (AKM ? 1 : 2) + NI * (BKM ? 1 : 2), MF = MI * NI;
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                if (reads && 2 * i < RD) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        Chunk<T> ca[A::L], cb[B::L];
        const T *ata[A::L], *atb[B::L];
        a.pointers(ata, tid);
        b.pointers(atb, tid);
        if (steps > 0) {
            a.fetch(ca, ata, 0, tid);
            b.fetch(cb, atb, 0, tid);
        }
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            a.store(ca, s, smem, tid);
            b.store(cb, s, smem + PA, tid);
            __syncthreads();
            if (s + 1 < steps) {
                a.fetch(ca, ata, s + 1, tid);
                b.fetch(cb, atb, s + 1, tid);
            }
            read(0, smem, 0);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk + 1 < KK) read((kk + 1) & 1, smem, kk + 1);
                multiply(kk & 1);
                interleave(kk + 1 < KK);
            }
        }
    }
    write_tile<T, MI, NI>(p, id, m0 + wm, n0 + wn, acc, smem, lane, wave);
}

// The same for fp32: every operand as three bf16 parts (split.hpp), a product as
// six, 128 x 128 outputs per workgroup of 2 x 2 waves, stages of 16 values.
// While a wave multiplies stage s, it reads the fragments of stage s + 1, splits
// stage s + 2 from registers into the LDS buffer that stage s has left, and
// loads stage s + 4, so a step has one barrier.  Bound by the matrix cores (six
// products at bf16's rate) with the vector instructions of the splitting beside
// them: 4096^3 190 to 204 TFLOP/s, where the fp32 matrix cores' peak is 157.
template <bool AKM, bool BKM>
__global__ __launch_bounds__(256, 2) void split_product_kernel(ProductArgs p)
{
    constexpr int BM = 128, BN = 128, KT = 16, MI = 2, NI = 2, NT = 256;
    using A = Operand<float, StageOf<BM, KT, AKM>, NT>;
    using B = Operand<float, StageOf<BN, KT, BKM>, NT>;
    constexpr int PA = A::S.bytes(), PB = B::S.bytes(), BUF = 3 * (PA + PB);
    static_assert(A::L == 1 && B::L == 1, "one slot per thread");
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2 * 64, wn = wave % 2 * 64;

    const uint32_t tm = (uint32_t)((p.M + BM - 1) / BM), tn = (uint32_t)((p.N + BN - 1) / BN);
    if (blockIdx.y && workgroup_id() >= tm * tn * p.splits) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, p.splits);
    const int64_t m0 = (int64_t)id.m * BM, n0 = (int64_t)id.n * BN, k0 = id.split * p.k_part;
    const int64_t kn = p.K - k0 < p.k_part ? p.K - k0 : p.k_part;
    const int steps = kn > 0 ? (int)((kn + KT - 1) / KT) : 0;
    const A a{static_cast<const float*>(p.a) + (AKM ? m0 * p.lda + k0 : k0 * p.lda + m0), p.lda,
              (int)(p.M - m0 < BM ? p.M - m0 : BM), kn, AKM ? k0 + kn : p.M};
    const B b{static_cast<const float*>(p.b) + (BKM ? n0 * p.ldb + k0 : k0 * p.ldb + n0), p.ldb,
              (int)(p.N - n0 < BN ? p.N - n0 : BN), kn, BKM ? k0 + kn : p.N};

    f16v acc[MI][NI];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    };
    clear();
    u4 fa[2][MI][3], fb[2][NI][3];
    auto read = [&](int set, const char* buf) {
#pragma unroll
        for (int q = 0; q < 3; ++q) {
#pragma unroll
            for (int j = 0; j < NI; ++j) fb[set][j][q] = B::frag(buf + 3 * PA + q * PB, wn + 32 * j, 0, lane);
#pragma unroll
            for (int i = 0; i < MI; ++i) fa[set][i][q] = A::frag(buf + q * PA, wm + 32 * i, 0, lane);
        }
    };
    auto multiply = [&](int set) {
        constexpr int QA[6] = {2, 0, 1, 1, 0, 0}, QB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int q = 0; q < 6; ++q)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mma<float>(fb[set][j][QB[q]], fa[set][i][QA[q]], acc[i][j]);
    };
    Chunk<float> ca[2][1], cb[2][1];
    const float *ata[1], *atb[1];
    a.pointers(ata, tid);
    b.pointers(atb, tid);
    auto fetch = [&](int s) {
        if (s >= steps) return;
        a.fetch(ca[s & 1], ata, s, tid);
        b.fetch(cb[s & 1], atb, s, tid);
    };
    auto store = [&](int s) {
        if (s >= steps) return;
        a.store(ca[s & 1], s, smem + (s & 1) * BUF, tid);
        b.store(cb[s & 1], s, smem + (s & 1) * BUF + 3 * PA, tid);
    };
    // Step s of parity s & 1 = set; plain: stages s + 2 and s + 4 are whole.
    auto step = [&](int s, auto set, auto plain) {
        char* const own = smem + set * BUF;
        read(set ^ 1, smem + (set ^ 1) * BUF);
        if constexpr (plain) {
            A::put(ca[set], own, tid);
            B::put(cb[set], own + 3 * PA, tid);
            a.fetch_whole(ca[set], ata);
            b.fetch_whole(cb[set], atb);
        } else {
            store(s + 2);
            fetch(s + 4);
        }
        multiply(set);
        if constexpr (plain) {
            // a product, then a read or two and what splitting takes
            constexpr int RD = 3 * (MI * (AKM ? 1 : 2) + NI * (BKM ? 1 : 2));
#pragma unroll
            for (int i = 0; i < 24; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i < 12) __builtin_amdgcn_sched_group_barrier(0x100, RD / 12, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                if (i % 4 == 3) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            }
        }
        __syncthreads();
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::true_type yes;
    constexpr std::false_type no;
    fetch(0);
    fetch(1);
    store(0);
    store(1);
    fetch(2);
    fetch(3);
    __syncthreads();
    read(0, smem);
    __syncthreads();  // stage 2 takes the place of stage 0
    const int whole = a.plain() && b.plain() ? (int)(kn / KT) : 0;  // whole stages
    int s = 0;
    for (; s + 5 < whole; s += 2) {
        step(s, even, yes);
        step(s + 1, odd, yes);
    }
    for (; s < steps; s += 2) {
        step(s, even, no);
        if (s + 1 < steps) step(s + 1, odd, no);
    }

    // Sums that are infinite or NaN, or that the parts cannot hold, again as fp32
    // products, operands straight from memory (this wave's tile).
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            acc[i][j] *= SPLIT_UNSCALE;
#pragma unroll
            for (int e = 0; e < 16; ++e) z = fmaf(acc[i][j][e], 0.f, z);
        }
    if (__ballot(z != 0.f)) {
        clear();
        for (int64_t k = lane >> 5; k - (lane >> 5) < kn; k += 2) {
            float va[MI], vb[NI];
#pragma unroll
            for (int i = 0; i < MI; ++i) va[i] = a.at(wm + 32 * i + (lane & 31), k);
#pragma unroll
            for (int j = 0; j < NI; ++j) vb[j] = b.at(wn + 32 * j + (lane & 31), k);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(vb[j], va[i], acc[i][j], 0, 0, 0);
        }
    }
    write_tile<float, MI, NI>(p, id, m0 + wm, n0 + wn, acc, smem, lane, wave);
}

// Joins the parts of a split contraction in a fixed order and finishes the
// outputs: bound by the read of the parts.  WAVES == 1: a thread for each group of
// four columns; few groups of many parts would keep too few loads in flight so, and
// WAVES == 4 has a workgroup take 64 groups, its four waves every fourth part each.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs p)
{
    __shared__ f4 part[4][WAVES == 4 ? 64 : 1];
    const int lane = threadIdx.x & 63, wave = WAVES == 4 ? threadIdx.x >> 6 : 0;
    const int64_t nq = (p.N + 3) / 4, plane = p.M * p.N;
    const int64_t i = WAVES == 4 ? workgroup_id() * 64ll + lane : workgroup_id() * 256ll + threadIdx.x;
    const int64_t m = i >> 32 ? i / nq : (int64_t)((uint32_t)i / (uint32_t)nq), n = (i - m * nq) * 4;
    const int have = p.N - n < 4 ? (int)(p.N - n) : 4;
    f4 v[1] = {f4{0.f, 0.f, 0.f, 0.f}};
    ProductArgs whole = p;
    whole.splits = 1;
    const Ends ends = load_ends<T>(whole, n);
    if (m < p.M) {
        const float* const q = p.partial + m * p.N + n;
#pragma unroll 8
        for (int s = wave; s < p.splits; s += WAVES) v[0] += load4(q + s * plane, have);
    }
    if constexpr (WAVES == 4) {
        part[wave][lane] = v[0];
        __syncthreads();
        if (wave) return;
        v[0] = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    }
    if (m < p.M) finish_rows<T, 1>(p, m, 1, n, v, ends);
}

// Few rows (16 MB at most): bound by the read of B, then by A, which every
// workgroup reads.  A workgroup streams 16 NS columns of B once, its eight waves an
// eighth of the contraction each, D stages ahead, and they join their sums in LDS.
// Matrix instructions of 16 x 16 outputs, B's columns as their rows.  1 x 1024 x
// 4096 bf16 4.2 us (launch and latency), 24 x 4096 x 4096 7.7 (the 34 MB of B
// partly from the last-level cache, 8 TB/s beyond the launch), 24 x 4096 x 4096
// fp32 17.

// The sums of the eight waves for the same outputs, joined in order and finished.
// Columns from `whole` on stand `shift` to the right of their place.
template <typename T, int MB, int NS>
__device__ inline void join_waves(const ProductArgs& p, int64_t n0, const f4 (&acc)[MB][NS], float* lds, int lane,
                                  int wave, int whole = 16 * NS, int shift = 0)
{
    constexpr int EW = 16 * NS + 4, PLANE = MB * 16 * EW;
    const int r = threadIdx.x / (4 * NS), c = 4 * (threadIdx.x % (4 * NS));
    const int64_t n = n0 + c;
    const Ends ends = load_ends<T>(p, n);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
            *reinterpret_cast<f4*>(lds + wave * PLANE + (16 * i + (lane & 15)) * EW + 16 * j + 4 * (lane >> 4)) =
                acc[i][j];
    __syncthreads();
    if (r >= 16 * MB || r >= p.M || n >= p.N) return;
    f4 v[1] = {f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const float* const at = lds + w * PLANE + r * EW;
        f4 t = *reinterpret_cast<const f4*>(at + c);
        if (c >= whole)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = at[c + e + shift < EW ? c + e + shift : EW - 1];
        v[0] += t;
    }
    finish_rows<T, 1>(p, r, 1, n, v, ends);
}

// 16-bit types.  B contiguous along the output is turned by the reads of LDS.
template <typename T, bool BKM, int MB>
__global__ __launch_bounds__(512, 2) void rows_kernel(ProductArgs p)
{
    constexpr int NS = BKM ? 1 : 2, D = MB == 4 ? (BKM ? 3 : 2) : BKM && MB == 1 ? 8 : 4;  // what the registers hold
    constexpr Stage S{32, 64, false};
    constexpr int OWN = MB * LINES + (BKM ? LINES : S.bytes()), JOIN = MB * 16 * (16 * NS + 4) * 4;
    __shared__ __align__(16) char smem[8 * (JOIN > OWN ? JOIN : OWN)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowsPart<64> part(p.N, p.K, 16 * NS, wave);
    const int64_t n0 = part.n0, k1 = part.k1;
    const int cols = part.cols;
    const T* const a = static_cast<const T*>(p.a);
    const T* const b = static_cast<const T*>(p.b) + (BKM ? n0 * p.ldb : n0);
    f4 acc[MB][NS];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    struct St {
        raw16 x[MB][2], w[2 * NS];
    };
    char* const own = smem + wave * OWN;
    char* const own_w = own + MB * LINES;
    Lines al[MB], bl;
#pragma unroll
    for (int i = 0; i < MB; ++i) al[i] = Lines(16 * i, p.M, p.lda, lane, T{});
    uint32_t bo[2 * NS];
    const int left = cols < 8 ? cols - 8 : 0;  // a piece that passes the last column lies further left
    if constexpr (BKM) {
        bl = Lines(0, cols, p.ldb, lane, T{});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 64 * j + lane, c = S.slot_row(e);
            bo[j] = (uint32_t)(S.slot_k(e) * p.ldb + (c < cols - 8 ? c : cols - 8) - left) * 2;
        }
    }
    auto load = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) al[i].load(f.x[i], a + k);
        if constexpr (BKM)
            bl.load(f.w, b + k);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) f.w[j] = load_at(b + k * p.ldb + left, bo[j]);
    };
    auto load_last = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::load_last(f.x[i], a, 16 * i, p.M, p.lda, k, k1, lane);
        if constexpr (BKM)
            Lines::load_last(f.w, b, 0, cols, p.ldb, k, k1, lane);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t kr = k + S.slot_k(64 * j + lane);
                f.w[j] = load16(b + (kr < k1 ? kr : k1 - 1) * p.ldb, S.slot_row(64 * j + lane), cols);
                if (kr >= k1) f.w[j] = raw16{0, 0, 0, 0};
            }
    };
    auto use = [&](St& f) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::write(f.x[i], own + i * LINES, lane);
        if constexpr (BKM)
            Lines::write(f.w, own_w, lane);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<raw16*>(own_w + (64 * j + lane) * 16) = f.w[j];
        wave_fence();
        raw16 w[NS][2], x[MB][2];
        if constexpr (BKM)
            Lines::read(w[0], own_w, lane);
        else
#pragma unroll
            for (int h = 0; h < NS; ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    typedef __attribute__((address_space(3))) s4 ls4;
                    struct {
                        s4 x, y;
                    } z{__builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4*)(own_w + frag16_byte(S, 16 * h, 32 * j, lane, 0))),
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4*)(own_w + frag16_byte(S, 16 * h, 32 * j, lane, 1)))};
                    w[h][j] = __builtin_bit_cast(raw16, z);
                }
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::read(x[i], own + i * LINES, lane);
        wave_fence();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int h = 0; h < NS; ++h) {
                    if constexpr (__is_same(T, _Float16))
                        acc[i][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            __builtin_bit_cast(h8, w[h][j]), __builtin_bit_cast(h8, x[i][j]), acc[i][h], 0, 0, 0);
                    else
                        acc[i][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(b8, w[h][j]), __builtin_bit_cast(b8, x[i][j]), acc[i][h], 0, 0, 0);
                }
    };
    part.template run<D, St>(load, load_last, use);
    if constexpr (BKM)
        join_waves<T, MB, NS>(p, n0, acc, reinterpret_cast<float*>(smem), lane, wave);
    else
        join_waves<T, MB, NS>(p, n0, acc, reinterpret_cast<float*>(smem), lane, wave, cols & ~7, 8 - (cols & 7));
}

// fp32, on the fp32 matrix cores (the memory is slower): value 16 j + 4 g + e of
// a stage of 32 in the e-th of four instructions.
template <bool BKM, int MB>
__global__ __launch_bounds__(512, 2) void rows_fp32_kernel(ProductArgs p)
{
    constexpr int NS = 1, D = MB == 4 ? 3 : BKM && MB == 1 ? 8 : 4;
    constexpr int OWN = (MB + (BKM ? 1 : 0)) * LINES, JOIN = MB * 16 * (16 * NS + 4) * 4;
    __shared__ __align__(16) char smem[8 * (JOIN > OWN ? JOIN : OWN)];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowsPart<32> part(p.N, p.K, 16 * NS, wave);
    const int64_t n0 = part.n0, k1 = part.k1;
    const int cols = part.cols;
    const float* const a = static_cast<const float*>(p.a);
    const float* const b = static_cast<const float*>(p.b) + (BKM ? n0 * p.ldb : n0);
    f4 acc[MB][NS];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i][0] = f4{0.f, 0.f, 0.f, 0.f};
    struct St {
        raw16 x[MB][2], w[2];
    };
    char* const own = smem + wave * OWN;
    const int col = r < cols ? r : cols - 1;
    Lines al[MB], bl;
#pragma unroll
    for (int i = 0; i < MB; ++i) al[i] = Lines(16 * i, p.M, p.lda, lane, 0.f);
    if constexpr (BKM) bl = Lines(0, cols, p.ldb, lane, 0.f);
    const uint32_t bo = (uint32_t)(4 * g * p.ldb + col) * 4;
    auto load = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) al[i].load(f.x[i], a + k);
        if constexpr (BKM)
            bl.load(f.w, b + k);
        else
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f.w[j][e] = *reinterpret_cast<const uint32_t*>(
                        reinterpret_cast<const char*>(b + (k + 16 * j + e) * p.ldb) + bo);
    };
    auto load_last = [&](St& f, int64_t k) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::load_last(f.x[i], a, 16 * i, p.M, p.lda, k, k1, lane);
        if constexpr (BKM)
            Lines::load_last(f.w, b, 0, cols, p.ldb, k, k1, lane);
        else
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t kr = k + 16 * j + 4 * g + e;
                    f.w[j][e] = __builtin_bit_cast(uint32_t, b[(kr < k1 ? kr : k1 - 1) * p.ldb + col]);
                    if (kr >= k1) f.w[j][e] = 0u;
                }
    };
    auto use = [&](St& f) {
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::write(f.x[i], own + i * LINES, lane);
        if constexpr (BKM) Lines::write(f.w, own + MB * LINES, lane);
        wave_fence();
        raw16 x[MB][2], w[2] = {f.w[0], f.w[1]};
        if constexpr (BKM) Lines::read(w, own + MB * LINES, lane);
#pragma unroll
        for (int i = 0; i < MB; ++i) Lines::read(x[i], own + i * LINES, lane);
        wave_fence();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f4, w[j])[e],
                                                                     __builtin_bit_cast(f4, x[i][j])[e], acc[i][0], 0, 0, 0);
    };
    part.template run<D, St>(load, load_last, use);
    join_waves<float, MB, NS>(p, n0, acc, reinterpret_cast<float*>(smem), lane, wave);
}

// Many rows and a short contraction: bound by the read of A and the write of y,
// and a tile of the kernels above has too few stages to hide its begin and end.
// So 128 columns of B stay in LDS (a panel, split for fp32), and each of eight
// waves streams blocks of 32 rows past it without barriers, A from memory
// straight into fragments, the next block's loads under the products of this one.
// The panel lies as [plane][slot][column] in 16-byte slots, read without bank
// conflicts; slot 2 kk + h has the 8 values of half-wave h in product group kk:
// 16 kk + 8 h + i, or for fp32 (whose 8 are two loads) 16 kk + 4 h + i and 8 on,
// so that a row's two lanes read neighbours.  131072 x 128 x 512 fp32: 120 us (2.8
// TB/s, and 145 TFLOP/s of products), 150 with bias and GELU, whose vector
// instructions the products do not hide; bf16 with bias 54 us, with bias and GELU 71
// (3.1 and 2.4 TB/s).
constexpr int PANEL = 128;
template <typename T, bool BKM, int KK, bool WHOLE>
__global__ __launch_bounds__(512, 2) void panel_kernel(ProductArgs p)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int P = F32 ? 3 : 1, C = F32 ? 2 : 1, NJ = PANEL / 32, PLANE = 2 * KK * PANEL * 16, EW = 32 + 4,
                  LINE = 128 / (16 * (int)sizeof(T)),  // product groups per line
                  PF = F32 ? LINE : KK;                // and those under way
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* const a = static_cast<const T*>(p.a);
    const T* const b = static_cast<const T*>(p.b);

    const uint32_t panels = (uint32_t)((p.N + PANEL - 1) / PANEL), t = xcd_run(blockIdx.x, gridDim.x);
    const int64_t n0 = (int64_t)(t % panels) * PANEL, stride = (int64_t)(gridDim.x / panels) * 8;
    const int K = (int)p.K;
    auto first = [&](int kk, int h, int c) { return 16 * kk + (F32 ? 4 * h + 8 * c : 8 * h); };
    float* const bl = reinterpret_cast<float*>(smem + P * PLANE);
    if (tid < PANEL) bl[tid] = p.bias && n0 + tid < p.N ? (float)static_cast<const T*>(p.bias)[n0 + tid] : 0.f;
    for (int i = tid; i < 2 * KK * PANEL; i += 512) {
        const int col = i % PANEL, kk = i / PANEL / 2, h = i / PANEL % 2;
        const int64_t n = n0 + col < p.N ? n0 + col : p.N - 1;  // (columns that do not exist are not written)
        Chunk<T> v;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (BKM) {
                v.v[c] = load16(b + n * p.ldb, first(kk, h, c), K);
                settle16<T>(v.v[c], first(kk, h, c), K);
            } else {
                T e[per16<T>];
#pragma unroll
                for (int u = 0; u < per16<T>; ++u) {
                    const int k = first(kk, h, c) + u;
                    e[u] = b[(k < K ? k : K - 1) * p.ldb + n];
                    if (k >= K) e[u] = (T)0.f;
                }
                __builtin_memcpy(&v.v[c], e, 16);
            }
        }
        if constexpr (F32) {
            u4 s[3];
            split_chunk(v, s);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<u4*>(smem + q * PLANE + i * 16) = s[q];
        } else {
            *reinterpret_cast<u4*>(smem + i * 16) = v.v[0];
        }
    }
    __syncthreads();

    const int64_t blocks = (p.M + 31) / 32;
    const int64_t b0 = (int64_t)(t / panels) * 8 + wave;
    if (b0 >= blocks) return;
    auto line = [&](int64_t blk) {
        const int64_t row = 32 * blk + (lane & 31);
        return a + (row < p.M ? row : p.M - 1) * p.lda;
    };
    const char* const mine = smem + (half * PANEL + (lane & 31)) * 16;
    float* const tile = bl + PANEL + wave * 32 * EW;
    Ends ends = load_ends<T>(p, p.N);  // (the generator's; the bias is in LDS)
    Chunk<T> x[PF];
    auto load = [&](const T* l, int kk) {
#pragma unroll
        for (int c = 0; c < C; ++c) x[kk % PF].v[c] = load16(l, first(kk, half, c), K);
    };
    auto fragment = [&](int kk, u4 (&to)[P]) {
        if constexpr (!WHOLE)
#pragma unroll
            for (int c = 0; c < C; ++c) settle16<T>(x[kk % PF].v[c], first(kk, half, c), K);
        if constexpr (F32) split_chunk(x[kk % PF], to);
        else to[0] = x[kk % PF].v[0];
    };
    {
        const T* const l = line(b0);
#pragma unroll
        for (int kk = 0; kk < PF; ++kk) load(l, kk);
    }
    for (int64_t blk = b0; blk < blocks; blk += stride) {
        const T *const now = line(blk), *const next = line(blk + stride < blocks ? blk + stride : blk);
        f16v acc[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
        u4 w[2][P], xs[2][P];
        auto read = [&](u4 (&to)[P], int kk, int j) {
#pragma unroll
            for (int q = 0; q < P; ++q)
                to[q] = *reinterpret_cast<const u4*>(mine + q * PLANE + (2 * kk * PANEL + 32 * j) * 16);
        };
        read(w[0], 0, 0);
        fragment(0, xs[0]);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk % LINE == LINE - 1)  // whole lines of memory at once
#pragma unroll
                for (int l = kk - LINE + 1; l <= kk; ++l) {
                    if (l + PF < KK) load(now, l + PF);
                    else load(next, l + PF - KK);
                }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int u = (kk * NJ + j) & 1;
                const bool last = j == NJ - 1;
                if (!last) read(w[u ^ 1], kk, j + 1);
                else if (kk + 1 < KK) read(w[u ^ 1], kk + 1, 0);
                if (last && kk + 1 < KK) fragment(kk + 1, xs[(kk + 1) & 1]);
                if constexpr (F32) {
                    constexpr int QW[6] = {0, 2, 1, 0, 1, 0}, QX[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
                    for (int q = 0; q < 6; ++q) acc[j] = mma<T>(w[u][QW[q]], xs[kk & 1][QX[q]], acc[j]);
                    if constexpr (WHOLE) {
                        // the next fragments' reads, and the splitting, between the products
#pragma unroll
                        for (int q = 0; q < 6; ++q) {
                            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                            if (q < 3) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                            if (last) __builtin_amdgcn_sched_group_barrier(0x002, 10, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                } else {
                    acc[j] = mma<T>(w[u][0], xs[kk & 1][0], acc[j]);
                }
            }
        }
        if constexpr (F32) {
            // sums that are infinite or NaN again as fp32 products, as above
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                acc[j] *= SPLIT_UNSCALE;
#pragma unroll
                for (int e = 0; e < 16; ++e) z = fmaf(acc[j][e], 0.f, z);
            }
            if (__ballot(z != 0.f)) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
                const T* const l = line(blk);
                for (int k0 = 0; k0 < K; k0 += 2) {
                    const int k = k0 + half;
                    const float xv = k < K ? (float)l[k] : 0.f;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int64_t n = n0 + 32 * j + (lane & 31);
                        const float wv = k < K && n < p.N ? (float)b[BKM ? n * p.ldb + k : k * p.ldb + n] : 0.f;
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(wv, xv, acc[j], 0, 0, 0);
                    }
                }
            }
        }
        // 32 columns at a time through LDS: 8 lanes hold a row's.  A block that is
        // not whole ends with a wait for all of its stores.
        auto turn = [&](const f16v& c, f4 (&v)[4]) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f4*>(tile + (lane & 31) * EW + 8 * g + 4 * half) =
                    f4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const f4*>(tile + ((lane >> 3) + 8 * r) * EW + 4 * (lane & 7));
        };
        const int64_t m = 32 * blk + (lane >> 3);
        f4 v[4];
        if (32 * blk + 32 <= p.M && n0 + PANEL <= p.N) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                turn(acc[j], v);
                ends.bias = *reinterpret_cast<const f4*>(bl + 32 * j + 4 * (lane & 7));
                finish_rows<T, 4, true>(p, m, 8, n0 + 32 * j + 4 * (lane & 7), v, ends);
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < NJ; ++j) {
                switch (j) {
                case 0: turn(acc[0], v); break;
                case 1: turn(acc[1], v); break;
                case 2: turn(acc[2], v); break;
                case 3: turn(acc[3], v); break;
                }
                const int64_t n = n0 + 32 * j + 4 * (lane & 7);
                ends.bias = *reinterpret_cast<const f4*>(bl + 32 * j + 4 * (lane & 7));
                if (n < p.N) finish_rows<T, 4>(p, m, 8, n, v, ends);
            }
            wait_direct();
        }
    }
}

// What a product of g is multiplied by: the dropout's 1 / (1 - p), and 1 / fit_slope.
// Both are left out of the 16-bit g, so that it is exact without an activation and
// with ReLU (dy or zero), and does not overflow where dx and dw do not: the slopes
// of GELU and SiLU are at most 1.13, which fp16 would not hold times its largest
// dy.  Otherwise g's one rounding is at most 2^-8 (bf16) or 2^-11 (fp16) of it.
constexpr float FIT_SLOPE = 0.875f;
template <typename T>
constexpr float fit_slope(int act)
{
    return __is_same(T, _Float16) && (act == CLIFF_ACT_GELU || act == CLIFF_ACT_SILU) ? FIT_SLOPE : 1.f;
}

// The pre-activations of four columns, in T, or in 8 bits with pre_groups scales a row
// (EIGHT).
template <typename T, bool EIGHT>
__device__ inline f4 load_pre(const DenseBackwardArgs& a, const float* pre_scale, int64_t pre_groups, int64_t r, int64_t c,
                              int have)
{
    if constexpr (EIGHT) {
        Integers<4> q;
        q.load(static_cast<const int8_t*>(a.pre) + r * a.ldp + c, have);
        const float s = pre_scale[r * pre_groups + (pre_groups > 1 ? c / CLIFF_INT8_GROUP : 0)];
        return f4{q.value(0, s), q.value(1, s), q.value(2, s), q.value(3, s)};
    } else {
        return load4(static_cast<const T*>(a.pre) + r * a.ldp + c, have);
    }
}

// g = keep dy f'(pre) fit_slope into g [M, N] (unless NULL), and the column sums
// of keep dy f'(pre) over a share of the rows into sums [part][N] (unless NULL); with
// EIGHT also keep dy f'(pre) in fp32 into g32 [M, N] (unless NULL).  A workgroup takes
// 256 columns; its four waves every fourth row each.  Bound by the vector instructions
// of f' and the generator: 8192 x 2048 bf16, GELU and dropout, 33 us (3 TB/s); 65536 x
// 512 fp32, SiLU, 87 us (4.6 TB/s, memory).
template <typename T, bool EIGHT>
__device__ inline void slope_rows(const DenseBackwardArgs& a, T* g, float* sums, int64_t rows_per_part,
                                  const float* pre_scale, int64_t pre_groups, float* g32)
{
    __shared__ f4 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = blockIdx.x * 256ll + 4 * lane;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.M ? r0 + rows_per_part : a.M;
    uint64_t key = 0;
    uint32_t step = 0;
    if (a.drop.rng) {
        key = (uint64_t)a.drop.rng[0];
        step = (uint32_t)a.drop.rng[1];
    }
    DropArgs keep = a.drop;
    keep.scale = 1.f;
    f4 t = {0.f, 0.f, 0.f, 0.f};
    const int have = a.N - c < 4 ? (int)(a.N - c) : 4;
    if (c < a.N) {
#pragma unroll 4
        for (int64_t r = r0 + wave; r < r1; r += 4) {
            f4 v = load4(static_cast<const T*>(a.dy) + r * a.lddy + c, have);
            if (a.act != CLIFF_ACT_NONE) slope4<sizeof(T) == 4>(a.act, v, load_pre<T, EIGHT>(a, pre_scale, pre_groups, r, c, have));
            if (keep.rng) drop4(keep, key, step, r, c, v);
            t += v;
            if (g) store4(g + r * a.N + c, v * fit_slope<T>(a.act), have);
            if constexpr (EIGHT)
                if (g32) store4(g32 + r * a.N + c, v, have);
        }
    }
    if (!sums) return;
    part[wave][lane] = t;
    __syncthreads();
    if (wave) return;
    t = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < a.N) sums[blockIdx.y * a.N + c + e] = t[e];
}

template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(DenseBackwardArgs a, T* g, float* sums, int64_t rows_per_part)
{
    slope_rows<T, false>(a, g, sums, rows_per_part, nullptr, 0, nullptr);
}
template <typename T>
__global__ __launch_bounds__(256) void slope_int8_kernel(DenseBackwardInt8Args a, T* g, float* sums,
                                                         int64_t rows_per_part, float* g32)
{
    slope_rows<T, true>(a.dense, g, sums, rows_per_part, a.pre_scale, a.pre_groups, g32);
}

// The weight's gradient from x in 8 bits: sum over rows of q (scale g), the integers q
// exactly in bf16 and scale g from g in fp32.  bf16, where g is rounded (GELU and SiLU),
// rounds scale g instead, so that the product has one rounded operand as from x in 16
// bits (both rounded, x and g: an error of 1.7 times the output's own rounding, not 1.4).
// fp16 takes scale g as two bf16 parts, for in fp16 it could leave the range, and fp32
// as three (split.hpp), three products instead of the six of two split operands.
// The scale goes with a row and 128 features, so a workgroup's tile has 128 of them (of
// 128 x 128 outputs, 2 x 2 waves).
//
// Both operands go through registers, two stages of 32 rows ahead, and are converted on
// their way to one of two LDS buffers; a step has one barrier.  Bound by two waves per
// SIMD that convert and multiply in turn (a quarter to a third of the matrix cores' rate):
// 8192 x 2048 x 2048 bf16 105 us, 65536 x 128 x 512 fp32 43; the conversion spread under
// the products took 120 us to 105, three workgroups on a compute unit spill (250).
template <typename T>
constexpr int weight_parts = sizeof(T) == 4 ? 3 : __is_same(T, _Float16) ? 2 : 1;
struct Int8Operand {
    const int8_t* q;
    int64_t ldq;
    const float* scale;
    int64_t groups;
    const float* g;  // [rows][N]
    int64_t ldg;
};
template <typename T, bool OI>
__global__ __launch_bounds__(256, 2) void weight_int8_kernel(ProductArgs p, Int8Operand o)
{
    constexpr int NT = 256, KT = 32, MI = 2, NI = 2, P = weight_parts<T>;
    using Tile = StageOf<128, KT, false>;
    using Op = Operand<__bf16, Tile, NT>;
    constexpr Stage S = Tile::s;
    constexpr int L = S.slots() / NT, BYTES = S.bytes(), BUF = (1 + P) * BYTES;
    extern __shared__ u4 smem4[];
    char* const smem = reinterpret_cast<char*>(smem4);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2 * 64, wn = wave % 2 * 64;
    const uint32_t tm = (uint32_t)((p.M + 127) / 128), tn = (uint32_t)((p.N + 127) / 128);
    if (blockIdx.y && workgroup_id() >= tm * tn * p.splits) return;
    const TileId id = tile_of(workgroup_id(), tm, tn, p.splits);
    // features and outputs of the layer: the rows and columns of dw, or the other way
    const int64_t k0 = (OI ? (int64_t)id.n : (int64_t)id.m) * 128, n0 = (OI ? (int64_t)id.m : (int64_t)id.n) * 128;
    const int64_t features = OI ? p.N : p.M, outputs = OI ? p.M : p.N;
    const int have_k = (int)(features - k0 < 128 ? features - k0 : 128), have_n = (int)(outputs - n0 < 128 ? outputs - n0 : 128);
    const int64_t r0 = id.split * p.k_part, rows = p.K - r0 < p.k_part ? p.K - r0 : p.k_part;
    const int steps = (int)((rows + KT - 1) / KT);
    const int8_t* const q = o.q + r0 * o.ldq + k0;
    const float* const g = o.g + r0 * o.ldg + n0;
    const float* const scale = o.scale + r0 * o.groups + (o.groups > 1 ? k0 / CLIFF_INT8_GROUP : 0);

    struct Fetched {
        Integers<8> q;
        f4 g[2];
        float s;
    };
    Fetched f[2][L];
    // Stages of whole rows in a whole tile have neither branches nor index arithmetic.
    const int whole = have_k == 128 && have_n == 128 ? (int)(rows / KT) : 0;
    const int8_t* at_q[L];
    const float *at_g[L], *at_s[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int e = i * NT + tid, c = S.slot_row(e), r = S.slot_k(e);
        at_q[i] = q + r * o.ldq + c;
        at_g[i] = g + r * o.ldg + c;
        at_s[i] = scale + r * o.groups;
    }
    auto fetch_one = [&](int s, Fetched (&to)[L], int i) {
        __builtin_memcpy(to[i].q.w, at_q[i] + s * (KT * o.ldq), 8);
        __builtin_memcpy(to[i].g, at_g[i] + s * (KT * o.ldg), 32);
        to[i].s = at_s[i][s * (KT * o.groups)];
    };
    auto fetch = [&](int s, Fetched (&to)[L]) {
        if (s >= steps) return;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (s < whole) {
                fetch_one(s, to, i);
                continue;
            }
            const int e = i * NT + tid, c = S.slot_row(e);
            const int64_t r = (int64_t)s * KT + S.slot_k(e), row = r < rows ? r : rows - 1;
            to[i].q.load(q + row * o.ldq + c, have_k - c);
            to[i].g[0] = load4(g + row * o.ldg + c, have_n - c);
            to[i].g[1] = load4(g + row * o.ldg + c + 4, have_n - c - 4);
            to[i].s = scale[row * o.groups];
            // (a row past the last one: zeros, whatever the last one has)
            if (r >= rows) to[i].g[0] = to[i].g[1] = f4{0.f, 0.f, 0.f, 0.f}, to[i].s = 0.f;
        }
    };
    // A slot's eight values of each operand, two at a time.
    struct Slot {
        b8 x, y[P];
        __device__ void convert(const Fetched& from, int pair)
        {
#pragma unroll
            for (int e = 2 * pair; e < 2 * pair + 2; ++e) {
                x[e] = (__bf16)from.q.value(e, 1.f);
                float v = from.g[e / 4][e % 4] * from.s;
                if constexpr (P == 3) v *= SPLIT_SCALE;
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    y[q][e] = (__bf16)v;
                    const float part = (float)y[q][e];
                    // (an infinity has no rest; three parts are found out by their NaN)
                    v = P == 2 && fabsf(part) == __builtin_inff() ? 0.f : v - part;
                }
            }
        }
        __device__ void put(char* to) const
        {
            *reinterpret_cast<b8*>(to) = x;
#pragma unroll
            for (int q = 0; q < P; ++q) *reinterpret_cast<b8*>(to + (1 + q) * BYTES) = y[q];
        }
    };
    auto put = [&](int s, const Fetched (&from)[L]) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            Slot slot;
#pragma unroll
            for (int pair = 0; pair < 4; ++pair) slot.convert(from[i], pair);
            slot.put(smem + (s & 1) * BUF + (i * NT + tid) * 16);
        }
    };
    f16v acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    fetch(0, f[0]);
    fetch(1, f[1]);
    put(0, f[0]);
    fetch(2, f[0]);
    __syncthreads();
    u4 fm[2][MI], fn[2][NI];
    constexpr int GROUPS = KT / 16 * P;  // of products: 16 rows, a part of scale g
    auto read = [&](int group, const char* buf) {
        const int set = group & 1, kk = group / P, q = group % P;
        const char* const from_m = buf + (OI ? (1 + q) * BYTES : 0);
        const char* const from_n = buf + (OI ? 0 : (1 + q) * BYTES);
#pragma unroll
        for (int j = 0; j < NI; ++j) fn[set][j] = Op::frag(from_n, wn + 32 * j, 16 * kk, lane);
#pragma unroll
        for (int i = 0; i < MI; ++i) fm[set][i] = Op::frag(from_m, wm + 32 * i, 16 * kk, lane);
    };
    // Step s, with the fetched stage s + 1; plain: that and stage s + 3 are whole.  Under
    // every product, the next group's fragments and a share of the conversion.
    auto step = [&](int s, Fetched (&next)[L], auto plain) {
        const char* const buf = smem + (s & 1) * BUF;
        char* const to = smem + ((s + 1) & 1) * BUF + tid * 16;
        if constexpr (!plain) {
            if (s + 1 < steps) put(s + 1, next);
            fetch(s + 3, next);
        }
        Slot slot;
        read(0, buf);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 4 * GROUPS; ++u) {
            const int group = u / 4, i = u / 2 % 2, j = u % 2;
            acc[i][j] = mma<__bf16>(fn[group & 1][j], fm[group & 1][i], acc[i][j]);
            if (u % 4 == 0 && group + 1 < GROUPS) read(group + 1, buf);
            if constexpr (plain) {
                if (u % P == 0) {
                    const int pair = u / P;  // of eight, of both slots
                    slot.convert(next[pair / 4], pair % 4);
                    if (pair % 4 == 3) {
                        slot.put(to + pair / 4 * NT * 16);
                        fetch_one(s + 3, next, pair / 4);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
    };
    static_assert(L == 2 && MI == 2 && NI == 2, "shares of the conversion");
    constexpr std::true_type yes;
    constexpr std::false_type no;
    int s = 0;
    for (; s + 4 < whole; s += 2) {
        step(s, f[1], yes);
        step(s + 1, f[0], yes);
    }
    for (; s < steps; s += 2) {
        step(s, f[1], no);
        if (s + 1 < steps) step(s + 1, f[0], no);
    }
    if constexpr (P == 3) {
        // Sums that are infinite or NaN, or that the parts cannot hold, again as fp32
        // products, operands straight from memory (this wave's tile).
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                acc[i][j] *= 1.0f / SPLIT_SCALE;
#pragma unroll
                for (int e = 0; e < 16; ++e) z = fmaf(acc[i][j][e], 0.f, z);
            }
        if (__ballot(z != 0.f)) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
            auto at = [&](bool left, int c, int64_t r) {  // an element of x or of g
                if (r >= rows || c >= (left ? have_k : have_n)) return 0.f;
                return left ? (float)q[r * o.ldq + c] * scale[r * o.groups] : g[r * o.ldg + c];
            };
            for (int64_t r = lane >> 5; r - (lane >> 5) < rows; r += 2) {
                float va[MI], vb[NI];
#pragma unroll
                for (int i = 0; i < MI; ++i) va[i] = at(!OI, wm + 32 * i + (lane & 31), r);
#pragma unroll
                for (int j = 0; j < NI; ++j) vb[j] = at(OI, wn + 32 * j + (lane & 31), r);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(vb[j], va[i], acc[i][j], 0, 0, 0);
            }
        }
    }
    write_tile<T, MI, NI>(p, id, (int64_t)id.m * 128 + wm, (int64_t)id.n * 128 + wn, acc, smem, lane, wave);
}

// x in 8 bits, as the product with g reads it.
template <typename T>
__global__ __launch_bounds__(256) void expand_kernel(DequantizeArgs a, uint32_t pieces, int64_t n)
{
    dequantize_rows<T>(a, workgroup_id() * 256ll + threadIdx.x, pieces, n);
}

// dbias: scale times the parts [part][N], joined in a fixed order: 64 columns per
// workgroup, every 16th part per wave.
template <typename T>
__global__ __launch_bounds__(1024) void bias_kernel(const float* sums, int parts, int64_t N, float scale, T* dbias)
{
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = workgroup_id() * 64ll + lane;
    float t = 0.f;
    if (c < N) {
#pragma unroll 8
        for (int i = wave; i < parts; i += 16) t += sums[i * N + c];
    }
    s[wave][lane] = t;
    __syncthreads();
    if (wave || c >= N) return;
    t = 0.f;
    for (int i = 0; i < 16; ++i) t += s[i][lane];
    dbias[c] = (T)(t * scale);
}

// How a product is cut: tiles of 256 x 256 or 128 x 128, and parts of the
// contraction.
struct Cut {
    bool large;
    int splits;
    int64_t k_part;
    double ns;  // what it is expected to take
};

// Times in ns, fitted to measured ones (MI355X; 31 products of 128 to 8008 rows
// and columns with 1 to 32 parts each, 12 % off on average; the cuts that they
// choose take 1 % longer than the best ones, 18 % at worst): of a stage with one
// workgroup on each compute unit and with as many as fit, and of a workgroup's
// begin and end.  The kernels wait for memory most of the time when they are
// alone, so a second workgroup costs less than the first.
struct TileTimes {
    int B, KT, fit;
    double alone, full, ends;
};
constexpr TileTimes T_DIRECT256{256, 64, 1, 1300, 1300, 10000}, T_DIRECT128{128, 64, 2, 600, 1150, 5800},
    T_STAGED128{128, 64, 2, 1100, 1550, 6300}, T_SPLIT128{128, 16, 2, 700, 1230, 8000};

Cut cut(int dtype, int64_t M, int64_t N, int64_t K, bool direct)
{
    const int64_t cus = std::max(device_cus(), 1);
    Cut best{false, 1, 0, 0};
    for (int large = 0; large <= (direct ? 1 : 0); ++large) {
        const TileTimes& t = large ? T_DIRECT256 : dtype == CLIFF_F32 ? T_SPLIT128 : direct ? T_DIRECT128 : T_STAGED128;
        const int64_t tiles = ceil_div(M, t.B) * ceil_div(N, t.B), steps = std::max<int64_t>(1, ceil_div(K, t.KT));
        for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}) {
            if (want > steps) break;
            const int64_t per = ceil_div(steps, want), splits = ceil_div(steps, per);
            const int64_t wgs = tiles * splits, rounds = wgs / (cus * t.fit), rest = wgs % (cus * t.fit);
            double ns = rounds * (per * t.full + t.ends);
            if (rest) ns += per * (rest <= cus ? t.alone : t.full) + t.ends;
            // the join: a launch, and the partial sums written and read
            if (splits > 1) ns += 4400 + (double)M * N * 4 * 2 * splits / 11700;
            if (best.ns == 0 || ns < best.ns) best = Cut{large != 0, (int)splits, per * t.KT, ns};
        }
    }
    return best;
}

// What the kernels of few rows are for: rows, row strides (32-bit offsets), and
// outputs (2^32 threads of a grid).
constexpr int64_t FEW_ROWS = 64, FEW_LD = 1 << 23, FEW_N = 1 << 26;

// The time in ns of few_rows, from bytes that a compute unit takes in, to choose
// between it and the tiles: every workgroup reads all of A, so that with a long
// contraction and little else to share it the parts of split tiles are ahead.  24 x
// 4096 x 4096 bf16: 7.7 us here, 13.8 in tiles; 24 x 8192 x 2048, B contiguous
// along the output: 21.3 and 14.3; 64 x 4096 x 1024 fp32: 25 and 19.
template <typename T, bool BKM>
double few_rows_ns(const ProductArgs& p)
{
    const int cols = BKM || sizeof(T) == 4 ? 16 : 32, rows = p.M <= 16 ? 16 : p.M <= 32 ? 32 : 64;
    const double rounds = std::max(1., (double)ceil_div(p.N, cols) / std::max(device_cus(), 1));
    return 3500 + rounds * (double)(p.K * (rows + cols) * (int64_t)sizeof(T)) / (sizeof(T) == 4 ? 57 : BKM ? 75 : 65);
}

// What a product of rows (y or dx) or a weight's gradient needs for its parts.
int64_t partial_bytes(int dtype, int64_t M, int64_t N, int64_t K)
{
    int64_t n = 0;
    for (int direct = 0; direct <= (dtype == CLIFF_F32 ? 0 : 1); ++direct) {
        const Cut c = cut(dtype, M, N, K, direct != 0);
        if (c.splits > 1) n = std::max(n, c.splits * M * N * 4);
    }
    return ceil_div(n, 256) * 256;
}

bool aligned_rows(const void* x, int64_t ld, int64_t width)
{
    return ((uintptr_t)x & 15) == 0 && ld % 8 == 0 && width % 8 == 0 && ld <= (1 << 21);
}

// Enqueues kernel k for tiles of B x B; its stages take `stage` bytes of LDS.
template <typename K, typename... More>
cliff_status run(K k, const char* name, int B, int threads, int stage, const ProductArgs& p, hipStream_t stream,
                 const More&... more)
{
    const int lds = std::max(stage, threads / 64 * 32 * (64 + 4) * 4);  // or what write_tile takes
    const int64_t wgs = ceil_div(p.M, B) * ceil_div(p.N, B) * p.splits;
    if (wgs >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    if (debug_enabled())
        fprintf(stderr, "cliffconv: product %lld x %lld x %lld, %s tiles of %d, %lld workgroups, %d splits\n",
                (long long)p.M, (long long)p.N, (long long)p.K, name, B, (long long)wgs, p.splits);
    hipLaunchKernelGGL(k, grid_of(wgs), dim3(threads), lds, stream, p, more...);
    return launched();
}

template <typename T, bool BKM>
cliff_status few_rows(const ProductArgs& p, hipStream_t stream)
{
    const int64_t wgs = ceil_div(p.N, BKM || sizeof(T) == 4 ? 16 : 32);
    if (debug_enabled())
        fprintf(stderr, "cliffconv: product %lld x %lld x %lld, few rows, %lld workgroups\n", (long long)p.M,
                (long long)p.N, (long long)p.K, (long long)wgs);
    const auto go = [&](auto k) {
        hipLaunchKernelGGL(k, dim3((unsigned)wgs), dim3(512), 0, stream, p);
        return launched();
    };
    if constexpr (sizeof(T) == 4)
        return p.M <= 16 ? go(rows_fp32_kernel<BKM, 1>) : p.M <= 32 ? go(rows_fp32_kernel<BKM, 2>) : go(rows_fp32_kernel<BKM, 4>);
    else
        return p.M <= 16 ? go(rows_kernel<T, BKM, 1>) : p.M <= 32 ? go(rows_kernel<T, BKM, 2>) : go(rows_kernel<T, BKM, 4>);
}

// Rows from which the panel kernel is level with the tiles or ahead (us, bias alone,
// panels and tiles; K 128, N 512: fp32 8192 rows 16.7 and 16.2, 16384 rows 19.2 and
// 22.1, 131072 rows 119 and 156; bf16 10.8 and 9.4, 11.8 and 11.5, 54 and 64.  K 64,
// N 256: ahead from 8192 rows.  K 128, N 128, one panel: behind by 1.5 up to 32768
// rows, ahead from 65536), the contraction whose panel fits LDS in fp32 (in 16 bits
// longer ones would; 131072 x 256 x 1024 bf16 takes the tiles 143), and its launch.
constexpr int64_t PANEL_ROWS = 16384;
constexpr int64_t PANEL_K = 128;

template <typename T, bool BKM>
cliff_status panel(const ProductArgs& p, hipStream_t stream)
{
    const int64_t panels = ceil_div(p.N, PANEL), cus = std::max(device_cus(), 1);
    const int64_t groups = std::min(std::max<int64_t>(1, cus / panels), ceil_div(p.M, 32 * 8));
    if (panels * groups >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    if (debug_enabled())
        fprintf(stderr, "cliffconv: product %lld x %lld x %lld, panels, %lld workgroups\n", (long long)p.M,
                (long long)p.N, (long long)p.K, (long long)(panels * groups));
    const auto go = [&](auto k, int KK) {
        const int lds = (sizeof(T) == 4 ? 3 : 1) * 2 * KK * PANEL * 16 + (PANEL + 8 * 32 * (32 + 4)) * 4;
        hipLaunchKernelGGL(k, dim3((unsigned)(panels * groups)), dim3(512), lds, stream, p);
        return launched();
    };
    const auto sized = [&](auto kk) {
        constexpr int KK = decltype(kk)::value;
        return p.K == 16 * KK ? go(panel_kernel<T, BKM, KK, true>, KK) : go(panel_kernel<T, BKM, KK, false>, KK);
    };
    if (p.K <= 64) return sized(std::integral_constant<int, 4>{});
    return sized(std::integral_constant<int, 8>{});
}

// Groups of four outputs from which a thread joins all of a group's parts: 1003 x
// 777 x 1531 bf16 (384,000 groups, 2 parts) in 21.8 us with it and 24.3 with four
// waves, 128 x 2048 x 512 fp32 (16,000 groups) in 19.9 and 17.4.
constexpr int64_t JOIN_GROUPS = 1 << 17;

template <typename T>
cliff_status join(const ProductArgs& p, hipStream_t stream)
{
    const int64_t groups = p.M * ceil_div(p.N, 4);
    const bool one = groups >= JOIN_GROUPS;
    const int64_t blocks = ceil_div(groups, one ? 256 : 64);
    if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
    hipLaunchKernelGGL((one ? join_kernel<T, 1> : join_kernel<T, 4>), grid_of(blocks), dim3(256), 0, stream, p);
    return launched();
}

// A product and, where its contraction is split, the join.
template <typename T, bool AKM, bool BKM>
cliff_status product(int dtype, ProductArgs p, hipStream_t stream)
{
    const bool direct = sizeof(T) == 2 && aligned_rows(p.a, p.lda, AKM ? p.K : p.M) &&
                        aligned_rows(p.b, p.ldb, BKM ? p.K : p.N);
    const Cut c = cut(dtype, p.M, p.N, p.K, direct);
    if constexpr (AKM) {
        if (p.M <= FEW_ROWS && p.K >= per16<T> && (BKM || p.N >= per16<T>) && p.lda <= FEW_LD && p.ldb <= FEW_LD &&
            p.N <= FEW_N && few_rows_ns<T, BKM>(p) < c.ns)
            return few_rows<T, BKM>(p, stream);
        if (p.M >= PANEL_ROWS && p.K <= PANEL_K && p.K >= per16<T>) return panel<T, BKM>(p, stream);
    }
    p.splits = c.splits;
    p.k_part = c.k_part;
    cliff_status s;
    if constexpr (sizeof(T) == 4) {
        s = run(split_product_kernel<AKM, BKM>, "split", 128, 256, 2 * 3 * 2 * 128 * 16 * 2, p, stream);
    } else {
        if (!direct)
            s = run(product_kernel<T, AKM, BKM, 128, 128, 2, 2, 64, false>, "staged", 128, 256, 2 * 128 * 64 * 2, p, stream);
        else if (c.large)
            s = run(product_kernel<T, AKM, BKM, 256, 256, 2, 4, 64, true>, "direct", 256, 512, 2 * 2 * 256 * 64 * 2, p, stream);
        else
            s = run(product_kernel<T, AKM, BKM, 128, 128, 2, 2, 64, true>, "direct", 128, 256, 2 * 2 * 128 * 64 * 2, p, stream);
    }
    return s != CLIFF_OK || p.splits == 1 ? s : join<T>(p, stream);
}

// Workspace of the backward pass: g, the bias's partial sums, partial products.
struct BackwardSpace {
    int64_t g, sums, partial, all;
    int parts;
};
BackwardSpace backward_space(int dtype, int64_t M, int64_t K, int64_t N)
{
    BackwardSpace w;
    const int64_t cols = ceil_div(N, 256);
    w.parts = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(M, 16), ceil_div(2048, cols)));
    w.g = 0;
    w.sums = ceil_div(M * N * (dtype == CLIFF_F32 ? 4 : 2), 256) * 256;
    w.partial = w.sums + ceil_div(w.parts * N * 4, 256) * 256;
    w.all = w.partial + std::max({partial_bytes(dtype, M, K, N), partial_bytes(dtype, K, N, M),
                                  partial_bytes(dtype, N, K, M)});
    return w;
}

}  // namespace

int64_t dense_workspace(int dtype, int64_t M, int64_t K, int64_t N) { return partial_bytes(dtype, M, N, K); }
int64_t dense_backward_workspace(int dtype, int64_t M, int64_t K, int64_t N)
{
    return backward_space(dtype, M, K, N).all;
}

cliff_status launch_dense(int dtype, const DenseArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        ProductArgs p{a.M, a.N, a.K, a.x, a.ldx, a.w, a.ldw, 1, 1.f, 0, static_cast<float*>(a.workspace),
                      a.bias, a.act, a.drop, a.residual, a.ldr, a.pre, a.ldp, a.y, a.ldy};
        return a.w_out_in ? product<T, true, true>(dtype, p, stream) : product<T, true, false>(dtype, p, stream);
    });
}

namespace {

// What follows the slopes: dbias from its partial sums, dx and dw from g.
template <typename T>
cliff_status finish_backward(int dtype, const DenseBackwardArgs& a, const BackwardSpace& w, const void* g, int64_t ldg,
                             hipStream_t stream)
{
    char* const ws = static_cast<char*>(a.workspace);
    float* const partial = reinterpret_cast<float*>(ws + w.partial);
    const float scale = a.drop.rng ? a.drop.scale : 1.f;
    cliff_status s = CLIFF_OK;
    if (a.dbias) {
        hipLaunchKernelGGL(bias_kernel<T>, grid_of(ceil_div(a.N, 64)), dim3(1024), 0, stream,
                           reinterpret_cast<float*>(ws + w.sums), w.parts, a.N, scale, static_cast<T*>(a.dbias));
        s = launched();
    }
    const DropArgs none{nullptr, 0, 1.f};
    auto plain = [&](int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* y, int64_t ldy,
                     void* out, int64_t ldo) {
        return ProductArgs{M, N, K, x, ldx, y, ldy, 1, scale / fit_slope<T>(a.act), 0, partial, nullptr,
                           CLIFF_ACT_NONE, none, nullptr, 0, nullptr, 0, out, ldo};
    };
    if (s == CLIFF_OK && a.dx && a.M) {
        const ProductArgs p = plain(a.M, a.K, a.N, g, ldg, a.w, a.ldw, a.dx, a.lddx);
        s = a.w_out_in ? product<T, true, false>(dtype, p, stream) : product<T, true, true>(dtype, p, stream);
    }
    if (s == CLIFF_OK && a.dw)  // in the order of w: [K, N] = x^T g or [N, K] = g^T x
        s = product<T, false, false>(dtype,
                                     a.w_out_in ? plain(a.N, a.K, a.M, g, ldg, a.x, a.ldx, a.dw, a.lddw)
                                                : plain(a.K, a.N, a.M, a.x, a.ldx, g, ldg, a.dw, a.lddw),
                                     stream);
    return s;
}

// A gradient from 8 bits has in its workspace, beside what dense_backward has, x in its
// type with this row stride, or (weight_int8_kernel) g in fp32.
int64_t expanded_ld(int64_t K) { return ceil_div(K, 8) * 8; }  // (16-bit types)

// Parts of the rows for weight_int8_kernel, by the times in ns of a workgroup's stage of
// 32 rows, alone on a compute unit and with a second one, and of its begin and end
// (MI355X, one, two and three parts of scale g; tiles that are not whole wait for their
// loads: 20000 x 300 x 300 bf16 75 us in 24 parts and 58 in 96).
struct StageTimes {
    double alone, full;
};
constexpr StageTimes T_WEIGHT[] = {{930, 1640}, {500, 760}, {760, 1230}}, T_WEIGHT_EDGES{2400, 3000};  // by cliff_dtype
Cut weight_cut(int dtype, int64_t M, int64_t K, int64_t N)
{
    const int64_t cus = std::max(device_cus(), 1), tiles = ceil_div(K, 128) * ceil_div(N, 128), steps = ceil_div(M, 32);
    const StageTimes& t = K % 128 || N % 128 ? T_WEIGHT_EDGES : T_WEIGHT[dtype];
    Cut best{false, 1, 0, 0};
    for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}) {
        if (want > steps) break;
        const int64_t per = ceil_div(steps, want), splits = ceil_div(steps, per);
        const int64_t wgs = tiles * splits, rounds = wgs / (cus * 2), rest = wgs % (cus * 2);
        double ns = rounds * (per * t.full + 6000);
        if (rest) ns += per * (rest <= cus ? t.alone : t.full) + 6000;
        if (splits > 1) ns += 4400 + (double)K * N * 4 * 2 * splits / 11700;
        if (best.ns == 0 || ns < best.ns) best = Cut{false, (int)splits, per * 32, ns};
    }
    return best;
}

// Whether dw comes of weight_int8_kernel: in fp32, and where g is rounded.
bool exact_integers(int dtype, int act) { return dtype == CLIFF_F32 || act == CLIFF_ACT_GELU || act == CLIFF_ACT_SILU; }

// dw from x in 8 bits and g in fp32.
template <typename T>
cliff_status weight_int8(int dtype, const DenseBackwardInt8Args& a, const float* g, int64_t ldg, float* partial, hipStream_t stream)
{
    const DenseBackwardArgs& d = a.dense;
    const Cut c = weight_cut(dtype, d.M, d.K, d.N);
    const int64_t M = d.w_out_in ? d.N : d.K, N = d.w_out_in ? d.K : d.N;
    const DropArgs none{nullptr, 0, 1.f};
    const ProductArgs p{M, N, d.M, nullptr, 0, nullptr, 0, c.splits, d.drop.rng ? d.drop.scale : 1.f, c.k_part, partial,
                        nullptr, CLIFF_ACT_NONE, none, nullptr, 0, nullptr, 0, d.dw, d.lddw};
    const Int8Operand o{static_cast<const int8_t*>(d.x), d.ldx, a.x_scale, a.x_groups, g, ldg};
    const int stage = 2 * 128 * 32 * 2 * (1 + weight_parts<T>);
    const cliff_status s = d.w_out_in ? run(weight_int8_kernel<T, true>, "8-bit", 128, 256, stage, p, stream, o)
                                      : run(weight_int8_kernel<T, false>, "8-bit", 128, 256, stage, p, stream, o);
    return s == CLIFF_OK && p.splits > 1 ? join<T>(p, stream) : s;
}

}  // namespace

cliff_status launch_dense_backward(int dtype, const DenseBackwardArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const BackwardSpace w = backward_space(dtype, a.M, a.K, a.N);
        char* const ws = static_cast<char*>(a.workspace);
        const bool change = a.act != CLIFF_ACT_NONE || a.drop.rng;
        cliff_status s = CLIFF_OK;
        if (a.dbias || (change && (a.dx || a.dw))) {
            hipLaunchKernelGGL(slope_kernel<T>, dim3((unsigned)ceil_div(a.N, 256), (unsigned)w.parts), dim3(256), 0,
                               stream, a, change && (a.dx || a.dw) ? reinterpret_cast<T*>(ws + w.g) : nullptr,
                               a.dbias ? reinterpret_cast<float*>(ws + w.sums) : nullptr, ceil_div(a.M, w.parts));
            s = launched();
        }
        if (s != CLIFF_OK) return s;
        return finish_backward<T>(dtype, a, w, change ? ws + w.g : a.dy, change ? a.N : a.lddy, stream);
    });
}

int64_t dense_backward_int8_workspace(int dtype, int64_t M, int64_t K, int64_t N)
{
    const Cut c = weight_cut(dtype, M, K, N);
    int64_t more = c.splits > 1 ? c.splits * K * N * 4 : 0;
    if (dtype != CLIFF_F32)  // g in fp32 and the parts, or x
        more = std::max(ceil_div(M * N * 4, 256) * 256 + more, M * expanded_ld(K) * 2);
    return backward_space(dtype, M, K, N).all + ceil_div(more, 256) * 256;
}

cliff_status launch_dense_backward_int8(int dtype, const DenseBackwardInt8Args& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        DenseBackwardArgs d = a.dense;
        const BackwardSpace w = backward_space(dtype, d.M, d.K, d.N);
        char *const ws = static_cast<char*>(d.workspace), *const more = ws + w.all;
        const bool change = d.act != CLIFF_ACT_NONE || d.drop.rng;
        const bool exact = d.dw && d.M && exact_integers(dtype, d.act);
        // g in the type, for dx and for dw where it is not in fp32 beside it
        const bool g = change && (d.dx || (d.dw && (!exact || sizeof(T) == 4)));
        float* const g32 = exact && sizeof(T) == 2 ? reinterpret_cast<float*>(more) : nullptr;
        cliff_status s = CLIFF_OK;
        if (d.dbias || g || g32) {
            hipLaunchKernelGGL(slope_int8_kernel<T>, dim3((unsigned)ceil_div(d.N, 256), (unsigned)w.parts), dim3(256),
                               0, stream, a, g ? reinterpret_cast<T*>(ws + w.g) : nullptr,
                               d.dbias ? reinterpret_cast<float*>(ws + w.sums) : nullptr, ceil_div(d.M, w.parts), g32);
            s = launched();
        }
        if (s == CLIFF_OK && exact) {
            const float* const from = g32 ? g32 : static_cast<const float*>(change ? ws + w.g : d.dy);
            char* const partial = g32 ? more + ceil_div(d.M * d.N * 4, 256) * 256 : more;
            s = weight_int8<T>(dtype, a, from, g32 || change ? d.N : d.lddy, reinterpret_cast<float*>(partial), stream);
            d.dw = nullptr;
        }
        if constexpr (sizeof(T) == 2)
            if (s == CLIFF_OK && d.dw && d.M) {  // x as the product with g reads it
                const int64_t ld = expanded_ld(d.K), pieces = ceil_div(d.K, per16<T>);
                const int64_t n = pieces * ceil_div(d.M, DEQUANTIZE_ROWS), blocks = ceil_div(n, 256);
                if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
                const DequantizeArgs x{d.M, d.K, a.x_groups, static_cast<const int8_t*>(d.x), d.ldx, a.x_scale, more, ld};
                hipLaunchKernelGGL(expand_kernel<T>, grid_of(blocks), dim3(256), 0, stream, x, (uint32_t)pieces, n);
                s = launched();
                d.x = x.y;
                d.ldx = ld;
            }
        if (s != CLIFF_OK) return s;
        return finish_backward<T>(dtype, d, w, change ? static_cast<const void*>(ws + w.g) : d.dy, change ? d.N : d.lddy, stream);
    });
}

}  // namespace cliff
