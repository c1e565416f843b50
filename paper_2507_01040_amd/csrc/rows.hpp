// Parts of the kernels that go over rows (layer norm, dropout): 16 bytes of a
// row at a time, and sums over the lanes of a wave; and of those that multiply few
// rows: how eight waves share and load the operands.
#pragma once

#include "dense_geom.hpp"
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

// E 8-bit integers of neighbouring columns, of which some may not exist (have < E),
// and the values that they stand for.
template <int E>
struct Integers {
    uint32_t w[E / 4];
    __device__ void load(const int8_t* p, int have)
    {
        if (have >= E) {
            __builtin_memcpy(w, p, E);
        } else {
#pragma unroll
            for (int i = 0; i < E / 4; ++i) w[i] = 0;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < have) w[e / 4] |= (uint32_t)(uint8_t)p[e] << 8 * (e % 4);
        }
    }
    __device__ float value(int e, float scale) const { return (float)(int8_t)(w[e / 4] >> 8 * (e % 4)) * scale; }
};

// Integers to the values that they stand for: piece i of n, the same 16 bytes of the
// output of each of DEQUANTIZE_ROWS rows.
constexpr int DEQUANTIZE_ROWS = 4;
template <typename T>
__device__ inline void dequantize_rows(const DequantizeArgs& a, int64_t i, uint32_t pieces, int64_t n)
{
    constexpr int E = per16<T>, ROWS = DEQUANTIZE_ROWS;
    if (i >= n) return;
    const int64_t g = n >> 32 ? i / pieces : (int64_t)((uint32_t)i / pieces), r0 = g * ROWS;
    const int64_t col = (i - g * pieces) * E;
    const int have = a.d - col < E ? (int)(a.d - col) : E;
    Integers<E> q[ROWS];
    float s[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = r0 + r < a.rows ? r0 + r : a.rows - 1;
        q[r].load(a.q + row * a.ldq + col, have);
        s[r] = a.scale[row * a.groups + (a.groups > 1 ? col / CLIFF_INT8_GROUP : 0)];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = q[r].value(e, s[r]);
        if (r0 + r < a.rows) store16(static_cast<T*>(a.y) + (r0 + r) * a.ldy + col, v, have);
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
    static_assert(N == 16 || N == 32 || N == 64, "lanes");
    v += dpp<0xb1>(v);   // neighbours
    v += dpp<0x4e>(v);   // pairs
    v += dpp<0x141>(v);  // halves of 8, mirrored
    v += dpp<0x140>(v);  // halves of 16, mirrored
    if constexpr (N > 16) {
        const uint32_t a = __builtin_bit_cast(uint32_t, v);
        const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
        const uint32_t s0 = s[0], s1 = s[1];
        v = __builtin_bit_cast(float, s0) + __builtin_bit_cast(float, s1);
    }
    if constexpr (N > 32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto t = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const uint32_t t0 = t[0], t1 = t[1];
        v = __builtin_bit_cast(float, t0) + __builtin_bit_cast(float, t1);
    }
    return v;
}

// The sums of v[0..R) over the TPR threads of a row, in every one of them: 16, 32
// or 64 lanes, or the whole workgroup of TPR threads (then through `lds`, R
// floats a wave, with one barrier; the caller alternates two of them).
template <int TPR, int R>
__device__ inline void row_sums(float (&v)[R], float* lds)
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = lane_sum<(TPR < 64 ? TPR : 64)>(v[r]);
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

// ---- rows in registers

constexpr int wg_threads(int TPR) { return TPR > 256 ? TPR : 256; }

template <typename T>
__device__ inline raw16 load_piece(const T* row, int col, int64_t d)
{
    return d < per16<T> ? load16_narrow(row, col, d) : load16(row, col, d);
}
template <typename T, int TPR, int R, int C>
__device__ inline void settle_rows(raw16 (&x)[R][C], int t, int64_t d)
{
    if (d < per16<T> || d == (int64_t)C * TPR * per16<T>) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) settle16<T>(x[r][c], (c * TPR + t) * per16<T>, d);
}

// The elements of a vector [d] from column col on.
template <typename T>
__device__ inline void load_vector(const T* v, int col, int64_t d, float* to)
{
    raw16 r = load_piece(v, col, d);
    if (d >= per16<T>) settle16<T>(r, col, d);
    unpack16<T>(r, to);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a row is spread: calls f<TPR, EL, R>() with the smallest spread that holds
// d elements.  16 lanes of a wave, a wave, or a workgroup per row.
// Sixteen waves per row hold too few registers for the gradient.
template <bool BACKWARD, typename F>
bool with_spread(int64_t d, F&& f)
{
    if (d <= 16 * 8) f.template operator()<16, 8, 4>();
    else if (d <= 16 * 16) f.template operator()<16, 16, 2>();
    else if (d <= 64 * 8) f.template operator()<64, 8, 4>();
    else if (d <= 64 * 16) f.template operator()<64, 16, 2>();
    else if (d <= 256 * 8) f.template operator()<256, 8, 4>();
    else if (d <= 256 * 16) f.template operator()<256, 16, 2>();
    else if (d <= 512 * 16) f.template operator()<512, 16, 1>();
    else if constexpr (BACKWARD) return false;
    else if (d <= 1024 * 16) f.template operator()<1024, 16, 1>();
    else return false;
    return true;
}

// ---- few rows of a product

// What the eight waves share: the workgroup's columns, and a wave's part of the
// contraction (whole stages of KT but for the last).
template <int KT>
struct RowsPart {
    int64_t n0, k0, k1;
    int cols;
    __device__ RowsPart(int64_t N, int64_t K, int columns, int wave)
    {
        n0 = (int64_t)xcd_run(blockIdx.x, gridDim.x) * columns;
        cols = (int)(N - n0 < columns ? N - n0 : columns);
        const int64_t part = (K + 8 * KT - 1) / (8 * KT) * KT;
        k0 = wave * part;
        k1 = k0 + part < K ? k0 + part : K;
    }
    // Calls load(stage, k) D stages ahead of use(stage).  While D more stages
    // exist, no branch stands between a stage's load and its use: at a load that
    // may not have been issued, the wait for an older one becomes a wait for all.
    // A part's last values, less than a stage, come last, by load_last(stage, k).
    template <int D, typename St, typename L, typename S, typename U>
    __device__ void run(L load, S load_last, U use) const
    {
        const int n = k1 > k0 ? (int)((k1 - k0) / KT) : 0;
        St f[D];
        int s = 0;
        if (n >= 2 * D) {
#pragma unroll
            for (int d = 0; d < D; ++d) load(f[d], k0 + d * KT);
            do {
#pragma unroll
                for (int d = 0; d < D; ++d) {
                    use(f[d]);
                    load(f[d], k0 + (int64_t)(s + D + d) * KT);
                }
                s += D;
            } while (s + 2 * D <= n);
        } else {
#pragma unroll
            for (int d = 0; d < D; ++d)
                if (d < n) load(f[d], k0 + d * KT);
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (s + d < n) use(f[d]);
            if (s + D + d < n) load(f[d], k0 + (int64_t)(s + D + d) * KT);
        }
#pragma unroll
        for (int d = 0; d < D - 1; ++d)
            if (s + D + d < n) use(f[d]);
        const int64_t k = k0 + (int64_t)n * KT;
        if (k >= k1) return;
        load_last(f[0], k);
        use(f[0]);
    }
};

// 16 bytes at a byte offset of a lane from an address of the wave.
template <typename T>
__device__ inline raw16 load_at(const T* base, uint32_t offset)
{
    raw16 r;
    __builtin_memcpy(&r, reinterpret_cast<const char*>(base) + offset, 16);
    return r;
}

// A wave's piece of LDS: lines of 128 bytes, 16 of a block, in pieces of 16 bytes.
// Loads put a line's eight pieces on neighbouring lanes, and LDS, without barriers,
// turns them into fragments: 16 lanes that read one piece of 16 lines meet every
// bank once.  (Fragments straight from memory have four neighbouring lanes on four
// lines, which the L1 cache serves one at a time where lines lie a multiple of 128
// bytes apart: 24 x 4096 x 4096 bf16 in 12.0 us instead of 7.7.)
struct Lines {
    uint32_t at[2];  // a lane's two pieces of a block of lines, in bytes from the first
    template <typename T>
    __device__ Lines(int64_t first, int64_t lines, int64_t ld, int lane, T)
    {
        for (int h = 0; h < 2; ++h) {
            const int64_t l = first + 8 * h + (lane >> 3);
            at[h] = (uint32_t)((l < lines ? l : lines - 1) * ld + per16<T> * (lane & 7)) * (uint32_t)sizeof(T);
        }
    }
    Lines() = default;
    template <typename T>
    __device__ void load(raw16 (&v)[2], const T* base) const
    {
        for (int h = 0; h < 2; ++h) v[h] = load_at(base, at[h]);
    }
    static __device__ int byte(int line, int piece) { return line * 128 + ((piece ^ (line >> 1 & 7)) << 4); }
    static __device__ void write(const raw16 (&v)[2], char* lds, int lane)
    {
        for (int h = 0; h < 2; ++h) *reinterpret_cast<raw16*>(lds + byte(8 * h + (lane >> 3), lane & 7)) = v[h];
    }
    static __device__ void read(raw16 (&v)[2], const char* lds, int lane)
    {
        for (int j = 0; j < 2; ++j) v[j] = *reinterpret_cast<const raw16*>(lds + byte(lane & 15, 4 * j + (lane >> 4)));
    }
    // The values before k1 of a stage that is not whole, from value k on; lines
    // that do not exist give way to the last one here too.
    template <typename T>
    static __device__ void load_last(raw16 (&v)[2], const T* x, int64_t first, int64_t lines, int64_t ld, int64_t k,
                                     int64_t k1, int lane)
    {
        for (int h = 0; h < 2; ++h) {
            const int64_t l = first + 8 * h + (lane >> 3), pos = k + per16<T> * (lane & 7);
            v[h] = load16(x + (l < lines ? l : lines - 1) * ld, pos, k1);
            settle16<T>(v[h], pos, k1);
        }
    }
};
constexpr int LINES = 16 * 128;  // bytes of a block

__device__ inline void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

}  // namespace cliff
