// Rows in 8 bits and back: for each row, or each 128 features of one,
//   scale = max(max |x| / 127, 2^-126),   q = the integer nearest to x / scale,
// ties to the even one, and x is q scale from then on.
//
// Bound by memory: x is read once, in 16-byte pieces that stay in registers from
// the maximum to the rounding.  A scale's features lie on the lanes of half a wave
// or less (GROUP) or on those that layer norm would use for the row.  16384 x 4096 bf16
// by 128 features 39 us (5.2 TB/s) and back 31 (6.6), 8192 x 4096 fp32 by rows 26 (6.4);
// 4 x 4096 bf16 3.6 us, a launch.  Rounding by reciprocal and magic number, one branch
// for eight values, took 52 us to 39 at 131072 x 512 bf16, where vector instructions
// were the bound.
#include <stdio.h>

#include <algorithm>

#include "rows.hpp"

namespace cliff {
namespace {

constexpr int GROUP = CLIFF_INT8_GROUP;

// The largest |v| of the pieces as the bits of a float: these are in the order of
// the values, infinities and NaN above all others.
template <int E>
__device__ inline uint32_t most_bits(const float (&v)[E], uint32_t m)
{
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

// What a row's values are divided by.  Infinities and NaN make the scale NaN (and
// the integers zero): all values that it stands for are NaN then.  The quotients
// stay below 127.5, and scale and reciprocal are normal numbers.
struct Scale {
    float s, inv;
    bool finite;
    __device__ explicit Scale(uint32_t most)
    {
        finite = most < 0x7f800000u;
        const float m = finite ? __builtin_bit_cast(float, most) : 0.f;
        // m / 127, rounded once: the remainder of a quotient that is within a unit in the
        // last place, times 1 / 127 rounded, gives the nearest float (Markstein 1990)
        constexpr float R = 1.0f / 127.0f;
        const float q = m * R;
        s = fmaf(fmaf(-q, 127.0f, m), R, q);
        s = s > 0x1p-126f ? s : 0x1p-126f;
        inv = finite ? reciprocal(s) : 0.f;
        if (!finite) s = __builtin_nanf("");
    }
    // The integer nearest to v / s.  v inv is within 3 2^-24 of the quotient, relative,
    // so that only quotients within 3e-5 of the middle between two integers can go to
    // the wrong one; the sign of v - (k + 1/2) s, which 64 bits hold, decides those.
    __device__ int nearest(float v) const
    {
        const float k = floorf(v * inv);
        const double t = (double)v - ((double)k + 0.5) * (double)s;
        const int i = (int)k;
        return t > 0.0 ? i + 1 : t < 0.0 ? i : i + (i & 1);
    }
};

// E integers of a row's columns from `col` on, of which `have` exist.  Nearly all are
// the low bytes of v inv + 1.5 2^23, whose last place is one; next to the middle
// between two integers (one group in a thousand) they are found one by one.
template <int E>
__device__ inline void store_q(int8_t* to, const float (&v)[E], const Scale& s, int have)
{
    constexpr float MAGIC = 0x1.8p23f;
    float off = 0.f;
    uint32_t m[E], w[E / 4];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float f = fmaf(v[e], s.inv, MAGIC);
        m[e] = __builtin_bit_cast(uint32_t, f);
        off = fmaxf(off, fabsf(fmaf(v[e], s.inv, MAGIC - f)));
    }
    if (off > 0.4999f) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (fabsf(fmaf(v[e], s.inv, MAGIC - __builtin_bit_cast(float, m[e]))) > 0.4999f) m[e] = (uint32_t)s.nearest(v[e]);
    }
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(m[4 * i + 3], m[4 * i + 2], 0x0c0c0400u),
                                     __builtin_amdgcn_perm(m[4 * i + 1], m[4 * i], 0x0c0c0400u), 0x05040100u);
        if (!s.finite) w[i] = 0;
    }
    if (have >= E) {
        __builtin_memcpy(to, w, E);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < have) to[e] = (int8_t)(w[e / 4] >> 8 * (e % 4));
    }
}

// The largest of m over each aligned group of N lanes, in every one of them.
template <int CTRL>
__device__ inline uint32_t dpp_most(uint32_t m)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true);
    return o > m ? o : m;
}
template <int N>
__device__ inline uint32_t lane_most(uint32_t m)
{
    static_assert(N == 16 || N == 32 || N == 64, "lanes");
    m = dpp_most<0xb1>(m);
    m = dpp_most<0x4e>(m);
    m = dpp_most<0x141>(m);
    m = dpp_most<0x140>(m);
    if constexpr (N > 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        const uint32_t s0 = s[0], s1 = s[1];
        m = s0 > s1 ? s0 : s1;
    }
    if constexpr (N > 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        const uint32_t s0 = s[0], s1 = s[1];
        m = s0 > s1 ? s0 : s1;
    }
    return m;
}

// A scale for each 128 features (or for a row of that many at most): a thread has
// the same 16 bytes of each of ROWS rows.
constexpr int ROWS = 4;
template <typename T>
__global__ __launch_bounds__(256) void quantize_groups_kernel(QuantizeArgs a, uint32_t pieces, int64_t n)
{
    constexpr int E = per16<T>, LANES = GROUP / E;
    // (lanes past the last one do its work again and write nothing)
    const int64_t own = workgroup_id() * 256ll + threadIdx.x, i = own < n ? own : n - 1;
    const int64_t g = n >> 32 ? i / pieces : (int64_t)((uint32_t)i / pieces), r0 = g * ROWS;
    const int p = (int)(i - g * pieces);
    const int64_t col = (int64_t)p * E, have = a.d - col;
    raw16 x[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = r0 + r < a.rows ? r0 + r : a.rows - 1;
        const T* const line = static_cast<const T*>(a.x) + row * a.ldx;
        x[r] = a.d < E ? load16_narrow(line, col, a.d) : load16(line, col, a.d);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float v[E];
        if (a.d >= E) settle16<T>(x[r], col, a.d);
        unpack16<T>(x[r], v);
        const Scale s(lane_most<LANES>(most_bits<E>(v, 0)));
        if (own >= n || r0 + r >= a.rows) continue;
        if (have > 0) store_q<E>(a.q + (r0 + r) * a.ldq + col, v, s, have < E ? (int)have : E);
        if (p % LANES == 0) a.scale[(r0 + r) * (pieces / LANES) + p / LANES] = s.s;
    }
}

// One scale for a row, in the registers of TPR threads as in layer norm.
template <typename T, int TPR, int EL, int R>
__global__ __launch_bounds__(wg_threads(TPR)) void quantize_row_kernel(QuantizeArgs a)
{
    constexpr int E = per16<T>, C = EL / E, G = wg_threads(TPR) / TPR, W = TPR / 64;
    __shared__ uint32_t lds[2][(W ? W : 1) * R];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * G * R; r0 < a.rows; r0 += (int64_t)gridDim.x * G * R, turn ^= 1) {
        const int64_t rg = r0 + (int64_t)g * R;
        raw16 x[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = rg + r < a.rows ? rg + r : a.rows - 1;
#pragma unroll
            for (int c = 0; c < C; ++c)
                x[r][c] = load_piece(static_cast<const T*>(a.x) + row * a.ldx, (c * TPR + t) * E, a.d);
        }
        settle_rows<T, TPR, R, C>(x, t, a.d);
        uint32_t most[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            most[r] = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[E];
                unpack16<T>(x[r][c], v);
                most[r] = most_bits<E>(v, most[r]);
            }
            most[r] = lane_most<(TPR < 64 ? 16 : 64)>(most[r]);
        }
        if constexpr (W > 1) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) lds[turn][(threadIdx.x >> 6) * R + r] = most[r];
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const uint32_t o = lds[turn][w * R + r];
                    most[r] = o > most[r] ? o : most[r];
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (rg + r >= a.rows) continue;
            const Scale s(most[r]);
            if (t == 0) a.scale[rg + r] = s.s;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E, have = (int)a.d - col;
                float v[E];
                unpack16<T>(x[r][c], v);
                if (have > 0) store_q<E>(a.q + (rg + r) * a.ldq + col, v, s, have);
            }
        }
    }
}

// Rows that do not fit the registers: read twice, by one workgroup.
constexpr int WIDE = 1024;
template <typename T>
__global__ __launch_bounds__(WIDE) void quantize_wide_kernel(QuantizeArgs a)
{
    constexpr int E = per16<T>;
    __shared__ uint32_t lds[2][WIDE / 64];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const T* const x = static_cast<const T*>(a.x) + r * a.ldx;
        uint32_t most = 0;
        for (int64_t c = (int64_t)threadIdx.x * E; c < a.d; c += WIDE * E) {
            raw16 p = load16(x, c, a.d);
            float v[E];
            settle16<T>(p, c, a.d);
            unpack16<T>(p, v);
            most = most_bits<E>(v, most);
        }
        most = lane_most<64>(most);
        if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = most;
        __syncthreads();
        for (int w = 0; w < WIDE / 64; ++w) most = lds[turn][w] > most ? lds[turn][w] : most;
        const Scale s(most);
        if (threadIdx.x == 0) a.scale[r] = s.s;
        for (int64_t c = (int64_t)threadIdx.x * E; c < a.d; c += WIDE * E) {
            raw16 p = load16(x, c, a.d);
            float v[E];
            settle16<T>(p, c, a.d);
            unpack16<T>(p, v);
            store_q<E>(a.q + r * a.ldq + c, v, s, a.d - c < E ? (int)(a.d - c) : E);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(DequantizeArgs a, uint32_t pieces, int64_t n)
{
    dequantize_rows<T>(a, workgroup_id() * 256ll + threadIdx.x, pieces, n);
}

template <typename T>
struct QuantizeRow {
    const QuantizeArgs& a;
    hipStream_t stream;
    template <int TPR, int EL, int R>
    void operator()()
    {
        // few rows: one each, for every compute unit has one
        const int64_t cus = std::max(device_cus(), 1), groups = wg_threads(TPR) / TPR;
        if (a.rows <= cus * groups * R)
            launch<TPR, EL, 1>();
        else
            launch<TPR, EL, R>();
    }
    template <int TPR, int EL, int R>
    void launch()
    {
        constexpr int per_pass = wg_threads(TPR) / TPR * R;
        const int64_t blocks = std::min<int64_t>(ceil_div(a.rows, per_pass), 1 << 20);
        if (debug_enabled())
            fprintf(stderr, "cliffconv: quantize %lld x %lld, %d threads per row, %lld workgroups\n",
                    (long long)a.rows, (long long)a.d, TPR, (long long)blocks);
        hipLaunchKernelGGL((quantize_row_kernel<T, TPR, EL, R>), dim3((unsigned)blocks), dim3(wg_threads(TPR)), 0,
                           stream, a);
    }
};

}  // namespace

cliff_status launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (a.groups == 1 && a.d > GROUP) {
            if (!with_spread<false>(a.d, QuantizeRow<T>{a, stream}))
                hipLaunchKernelGGL(quantize_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)),
                                   dim3(WIDE), 0, stream, a);
            return launched();
        }
        const int64_t pieces = a.groups * (GROUP / per16<T>);
        const int64_t n = pieces * ceil_div(a.rows, ROWS), blocks = ceil_div(n, 256);
        if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
        if (debug_enabled())
            fprintf(stderr, "cliffconv: quantize %lld x %lld in groups, %lld workgroups\n", (long long)a.rows,
                    (long long)a.d, (long long)blocks);
        hipLaunchKernelGGL(quantize_groups_kernel<T>, grid_of(blocks), dim3(256), 0, stream, a, (uint32_t)pieces, n);
        return launched();
    });
}

cliff_status launch_dequantize(int dtype, const DequantizeArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t pieces = ceil_div(a.d, per16<T>);
        const int64_t n = pieces * ceil_div(a.rows, DEQUANTIZE_ROWS), blocks = ceil_div(n, 256);
        if (blocks >= (int64_t)1 << 31) return CLIFF_EUNSUPPORTED;
        if (debug_enabled())
            fprintf(stderr, "cliffconv: dequantize %lld x %lld, %lld workgroups\n", (long long)a.rows, (long long)a.d,
                    (long long)blocks);
        hipLaunchKernelGGL(dequantize_kernel<T>, grid_of(blocks), dim3(256), 0, stream, a, (uint32_t)pieces, n);
        return launched();
    });
}

}  // namespace cliff
