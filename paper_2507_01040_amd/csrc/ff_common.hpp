// Shared parts of the feed-forward operators (cliffconv_ff.h): types, the
// pointwise activations, the dropout generator, and what their launchers take.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

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

struct QuantizeArgs {
    int64_t rows, d, groups;  // groups: scales per row
    const void* x;
    int64_t ldx;
    int8_t* q;
    int64_t ldq;
    float* scale;
};

struct DequantizeArgs {
    int64_t rows, d, groups;
    const int8_t* q;
    int64_t ldq;
    const float* scale;
    void* y;
    int64_t ldy;
};

struct DenseInt8Args {
    int64_t M, K, N;
    const int8_t* x;
    int64_t ldx;
    const float* x_scale;
    const int8_t* w;
    int64_t ldw;
    const float* w_scale;
    const void* bias;
    int act;
    const void* residual;
    int64_t ldr;
    void* y;
    int64_t ldy;
    void* workspace;
};

// x and pre of `dense` in 8 bits, with x_groups and pre_groups scales per row.
struct DenseBackwardInt8Args {
    DenseBackwardArgs dense;
    const float* x_scale;
    int64_t x_groups;
    const float* pre_scale;
    int64_t pre_groups;
};

struct BlockNormArgs {
    int64_t rows, d;
    const void* x;
    int64_t ldx;
    const void* residual;
    int64_t ldr;
    const void* gate;  // [gates, d], each for rows / gates rows; gates 0: none
    int64_t gates;
    float scale, eps;
    bool after, before, rms;
    const void *weight, *bias, *next_weight, *next_bias;
    void* out;
    int64_t ldo;
    void* normed;
    int64_t ldn;
    float* stats;  // [4, rows]
};

struct BlockNormBackwardArgs {
    int64_t rows, d;
    const void* dout;
    int64_t lddo;
    const void* dnormed;
    int64_t lddn;
    const void* x;
    int64_t ldx;
    const void* out;
    int64_t ldo;
    const float* stats;
    const void* gate;
    int64_t gates;
    float scale;
    bool after, rms;
    const void *weight, *bias, *next_weight;
    void* dx;
    int64_t lddx;
    void* dresidual;
    int64_t lddr;
    void *dgate, *dweight, *dbias, *dnext_weight, *dnext_bias;
    void* workspace;
};

// ---- checks of a call's arguments (host)

constexpr int64_t MAX_SIZE = ((int64_t)1 << 31) - 1;  // of a width or row count
constexpr int64_t MAX_SPAN = (int64_t)1 << 40;        // elements from a matrix's first to its last

inline bool valid_dtype(int t) { return t >= CLIFF_F32 && t <= CLIFF_F16; }
inline int64_t size_of(int dtype) { return dtype == CLIFF_F32 ? 4 : 2; }

// A matrix, vector (one row) or workspace of a call.
struct Mat {
    const void* p;
    int64_t rows, cols, ld, elem;
};

inline bool bad_shape(const Mat& m)
{
    if (!m.p) return false;
    if (m.ld < m.cols) return true;
    return m.rows > 0 && (m.rows - 1) > (MAX_SPAN - 1 - m.cols) / m.ld;
}

inline bool misaligned(const Mat& m) { return ((uintptr_t)m.p & (uintptr_t)(m.elem - 1)) != 0; }

inline bool overlaps(const Mat& a, const Mat& b)
{
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.cols < 1 || b.cols < 1) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    const uintptr_t a1 = a0 + (uintptr_t)(((a.rows - 1) * a.ld + a.cols) * a.elem);
    const uintptr_t b1 = b0 + (uintptr_t)(((b.rows - 1) * b.ld + b.cols) * b.elem);
    if (a1 <= b0 || b1 <= a0) return false;
    const uintptr_t step = (uintptr_t)(a.ld * a.elem);
    if (step != (uintptr_t)(b.ld * b.elem)) return true;
    // one row stride: columns of b begin `off` bytes after a's, modulo the
    // stride, and end before a's begin again
    const uintptr_t off = b0 >= a0 ? (b0 - a0) % step : (step - (a0 - b0) % step) % step;
    return off < (uintptr_t)(a.cols * a.elem) || off + (uintptr_t)(b.cols * b.elem) > step;
}

inline bool same(const Mat& a, const Mat& b) { return a.p == b.p && a.ld == b.ld && a.elem == b.elem; }

// `out` against what it must not overlap; those in `may_equal` may be the same matrix.
inline bool clashes(const Mat& out, std::initializer_list<Mat> others, std::initializer_list<Mat> may_equal = {})
{
    for (const Mat& m : others)
        if (overlaps(out, m)) return true;
    for (const Mat& m : may_equal)
        if (!same(out, m) && overlaps(out, m)) return true;
    return false;
}

inline bool any_bad_shape(std::initializer_list<Mat> ms)
{
    for (const Mat& m : ms)
        if (bad_shape(m)) return true;
    return false;
}

inline bool any_misaligned(std::initializer_list<Mat> ms)
{
    for (const Mat& m : ms)
        if (misaligned(m)) return true;
    return false;
}

inline bool valid_drop(const cliff_dropout_desc* d)
{
    return !d || (d->p >= 0.0 && d->p <= 1.0 && (d->p == 0.0 || d->rng));
}

inline DropArgs to_args(const cliff_dropout_desc* d)
{
    DropArgs a{nullptr, 0, 1.f};
    if (!d || d->p == 0.0) return a;
    a.scale = d->p < 1.0 ? (float)(1.0 / (1.0 - d->p)) : 0.f;
    const double t = nearbyint(d->p * 4294967296.0);
    if (t < 1.0) return a;  // no word is below it
    a.rng = d->rng;
    a.last = (uint32_t)(t - 1.0);
    return a;
}

inline Mat vec(const void* p, int64_t n, int64_t elem) { return Mat{p, 1, n, n, elem}; }
inline Mat rng_of(const DropArgs& d) { return vec(d.rng, 2, 8); }

inline cliff_status check_workspace(const void* p, int64_t have, int64_t need)
{
    if (need == 0) return CLIFF_OK;
    if (!p || have < need) return CLIFF_ESCRATCH;
    return ((uintptr_t)p & 15u) ? CLIFF_EALIGN : CLIFF_OK;
}

// Widths and row counts, and the dense matrices of them (workspaces too).
inline bool valid_dense_sizes(int64_t M, int64_t K, int64_t N)
{
    return M >= 0 && M <= MAX_SIZE && K >= 1 && K <= MAX_SIZE && N >= 1 && N <= MAX_SIZE &&
           M * K < MAX_SPAN && M * N < MAX_SPAN && K * N < MAX_SPAN;
}

// ---- launches

// Launchers (the arguments are checked): dtype is a cliff_dtype.
cliff_status launch_dense(int dtype, const DenseArgs& a, hipStream_t stream);
int64_t dense_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status launch_dense_backward(int dtype, const DenseBackwardArgs& a, hipStream_t stream);
int64_t dense_backward_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status launch_layer_norm(int dtype, const NormArgs& a, hipStream_t stream);
cliff_status launch_layer_norm_backward(int dtype, const NormBackwardArgs& a, hipStream_t stream);
int64_t layer_norm_backward_workspace(int dtype, int64_t rows, int64_t d);
cliff_status launch_dropout(int dtype, const DropoutArgs& a, hipStream_t stream);
cliff_status launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t stream);
cliff_status launch_dequantize(int dtype, const DequantizeArgs& a, hipStream_t stream);
cliff_status launch_dense_int8(int dtype, const DenseInt8Args& a, hipStream_t stream);
int64_t dense_int8_workspace(int64_t M, int64_t K, int64_t N);
cliff_status launch_dense_backward_int8(int dtype, const DenseBackwardInt8Args& a, hipStream_t stream);
int64_t dense_backward_int8_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status launch_block_norm(int dtype, const BlockNormArgs& a, hipStream_t stream);
cliff_status launch_block_norm_backward(int dtype, const BlockNormBackwardArgs& a, hipStream_t stream);
int64_t block_norm_backward_workspace(int dtype, int64_t rows, int64_t d, int64_t gates);

inline cliff_status launched()
{
    return hipGetLastError() == hipSuccess ? CLIFF_OK : CLIFF_EDEVICE;
}

// A grid of n workgroups, and a workgroup's place in it.  HIP takes fewer than
// 2^32 threads along an axis, so that wide grids have rows; the last row can pass
// n, and workgroups there have nothing to do.
constexpr int64_t GRID_ROW = 1 << 16;
inline dim3 grid_of(int64_t n)
{
    return n <= GRID_ROW ? dim3((unsigned)n) : dim3((unsigned)GRID_ROW, (unsigned)((n + GRID_ROW - 1) / GRID_ROW));
}
__device__ inline uint32_t workgroup_id() { return blockIdx.y * (uint32_t)GRID_ROW + blockIdx.x; }

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

// a ^ b ^ c, in one instruction
__host__ __device__ inline uint32_t xor3(uint32_t a, uint32_t b, uint32_t c)
{
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
#else
    return a ^ b ^ c;
#endif
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
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c1 = (uint32_t)b;
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// 1 / v to the last bit or two
__device__ inline float reciprocal(float v) { return __builtin_amdgcn_rcpf(v); }

// Phi(v), and e = exp(-v^2 / 2) beside it: Phi(-|v|) = e R(|v|), where R falls
// smoothly from 1/2 and is a polynomial in t = 1 / (1 + 0.3 |v|) without
// constant term, fitted to the least relative error (1.5e-7 over the whole
// axis, 5e-7 as evaluated), so that small values of the left tail keep their
// digits.  FINE: what the exponent's rounding takes from e (4e-6 of it at |v| =
// 12) is put back; 16-bit results do not show it.
template <bool FINE>
__device__ inline float gelu_cdf(float v, float& e)
{
    const float a = fminf(fabsf(v), 16.f);  // e is zero there
    const float t = reciprocal(fmaf(0.3f, a, 1.0f));
    constexpr float C = -0.72134752f, C_REST = -9.62981495e-9f;  // -log2(e) / 2 = C + C_REST
    const float s = a * a, x = s * C;
    e = __builtin_amdgcn_exp2f(x);
    if constexpr (FINE) e = fmaf(e, fmaf(fmaf(a, a, -s), C, fmaf(s, C_REST, fmaf(s, C, -x))) * 0.69314718f, e);
    float r = fmaf(0.0356758006f, t, -0.157207165f);
    r = fmaf(r, t, 0.206360237f);
    r = fmaf(r, t, -0.0536895875f);
    r = fmaf(r, t, 0.128564652f);
    r = fmaf(r, t, 0.099912607f);
    r = fmaf(r, t, 0.120754093f);
    r = fmaf(r, t, 0.11962929f);
    r *= t * e;
    return v < 0.f ? r : 1.0f - r;
}

// 1 / (1 + exp(-v)), and what it lacks to 1, as e / (1 + e) on one side of zero and
// 1 / (1 + e) on the other, e = exp(-|v|): nothing overflows or cancels, and values
// of the left tail keep their digits down to the smallest ones.  FINE: what the
// exponent's rounding takes from e (4e-6 of it at |v| = 80) is put back; 16-bit
// results do not show it.
template <bool FINE>
__device__ inline float logistic(float v, float& lacks)
{
#pragma clang fp contract(off)  // x is what the exponential is taken of
    const float a = fminf(fabsf(v), 128.f);  // e is zero there
    constexpr float C = -1.44269502f, C_REST = -1.92596299e-8f;  // -log2(e) = C + C_REST
    const float x = a * C;
    float e = exp2f(x);
    if constexpr (FINE) e = fmaf(e, fmaf(a, C_REST, fmaf(a, C, -x)) * 0.69314718f, e);
    const float r = reciprocal(1.0f + e), er = e * r;
    lacks = v < 0.f ? r : er;
    return v < 0.f ? er : r;
}

template <bool FINE>
__device__ inline float activate(int act, float v)
{
    float e;
    switch (act) {
    case CLIFF_ACT_RELU: return v <= 0.f ? 0.f : v;  // NaN stays
    case CLIFF_ACT_GELU: return v * gelu_cdf<FINE>(v, e);
    case CLIFF_ACT_SILU: return v * logistic<FINE>(v, e);
    }
    return v;
}

template <bool FINE>
__device__ inline float activate_slope(int act, float v)
{
    float e;
    switch (act) {
    case CLIFF_ACT_RELU: return v > 0.f ? 1.f : v <= 0.f ? 0.f : v;  // NaN stays
    case CLIFF_ACT_GELU: {
        const float c = gelu_cdf<FINE>(v, e);
        return fmaf(v * 0.39894228040143268f, e, c);
    }
    case CLIFF_ACT_SILU: {
        const float s = logistic<FINE>(v, e);
        return s * fmaf(v, e, 1.0f);
    }
    }
    return 1.f;
}

// ---- four neighbouring columns

typedef float f4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Vec4 {
    typedef T t __attribute__((ext_vector_type(4)));
};

// Four neighbouring columns, of which some may not exist (have < 4).
template <typename T>
__device__ inline f4 load4(const T* p, int have)
{
    typename Vec4<T>::t v;
    if (have >= 4) {
        __builtin_memcpy(&v, p, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = (T)0.f;
            if (e < have) v[e] = p[e];
        }
    }
    return __builtin_convertvector(v, f4);
}
template <typename T>
__device__ inline void store4(T* p, const f4& v, int have)
{
    const typename Vec4<T>::t t = __builtin_convertvector(v, typename Vec4<T>::t);
    if (have >= 4) {
        __builtin_memcpy(p, &t, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) p[e] = t[e];
    }
}

template <bool FINE>
__device__ inline void activate4(int act, f4& v)
{
    switch (act) {
#define EACH(A)                                      \
    case A:                                          \
        for (int e = 0; e < 4; ++e) v[e] = activate<FINE>(A, v[e]); \
        break;
        EACH(CLIFF_ACT_RELU)
        EACH(CLIFF_ACT_GELU)
        EACH(CLIFF_ACT_SILU)
#undef EACH
    }
}
template <bool FINE>
__device__ inline void slope4(int act, f4& v, const f4& pre)
{
    switch (act) {
#define EACH(A)                                                  \
    case A:                                                      \
        for (int e = 0; e < 4; ++e) v[e] *= activate_slope<FINE>(A, pre[e]); \
        break;
        EACH(CLIFF_ACT_RELU)
        EACH(CLIFF_ACT_GELU)
        EACH(CLIFF_ACT_SILU)
#undef EACH
    }
}
__device__ inline void drop4(const DropArgs& d, uint64_t key, uint32_t step, int64_t r, int64_t c, f4& v)
{
    const Words w = philox(key, step, (uint32_t)(c >> 2), r);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w.w[e] <= d.last ? 0.f : v[e] * d.scale;
}

// ---- 16 bytes of a row

typedef uint32_t raw16 __attribute__((ext_vector_type(4)));

template <typename T>
constexpr int per16 = 16 / (int)sizeof(T);  // elements in them

// The 16 bytes from element pos of a line on (aligned to an element only), of a
// line whose elements before `end` may be read, in two steps, so that many loads
// can be under way: load16, and settle16 where the value is used.  A piece that
// passes the end is loaded from further left, where the line has it whole, and
// shifted; elements that do not exist become zeros.  The line has 16 bytes or
// more before its end; load16_narrow is for those that have not.
template <typename T>
__device__ inline raw16 load16(const T* line, int64_t pos, int64_t end)
{
    raw16 r;
    __builtin_memcpy(&r, line + (pos < end - per16<T> ? pos : end - per16<T>), 16);
    return r;
}
template <typename T>
__device__ inline void settle16(raw16& r, int64_t pos, int64_t end)
{
    constexpr int E = per16<T>;
    const int64_t over = pos + E - end;  // elements past the end
    if (over <= 0) return;
    const int s = over < E ? (int)over * 8 * (int)sizeof(T) : 128;
    uint64_t lo = r[0] | (uint64_t)r[1] << 32, hi = r[2] | (uint64_t)r[3] << 32;
    lo = s >= 128 ? 0 : s >= 64 ? hi >> (s - 64) : lo >> s | hi << (64 - s);
    hi = s >= 64 ? 0 : hi >> s;
    r = raw16{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
template <typename T>
__device__ inline raw16 load16_narrow(const T* line, int64_t pos, int64_t end)
{
    constexpr int E = per16<T>;
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        t[e] = (T)0.f;
        if (pos + e < end) t[e] = line[pos + e];
    }
    raw16 r;
    __builtin_memcpy(&r, t, 16);
    return r;
}

}  // namespace cliff
