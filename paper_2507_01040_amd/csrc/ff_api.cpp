// C ABI of the feed-forward operators (cliffconv_ff.h): argument checks and
// dispatch.  No device memory is allocated here; every call only enqueues
// kernels on the caller's stream.
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "cliffconv_ff.h"
#include "ff_common.hpp"

namespace {

using namespace cliff;

constexpr int64_t MAX_SIZE = ((int64_t)1 << 31) - 1;  // of a width or row count
constexpr int64_t MAX_SPAN = (int64_t)1 << 40;        // elements from a matrix's first to its last

bool valid_dtype(int t) { return t >= CLIFF_F32 && t <= CLIFF_F16; }
int64_t size_of(int dtype) { return dtype == CLIFF_F32 ? 4 : 2; }

// A matrix, vector (one row) or workspace of a call.
struct Mat {
    const void* p;
    int64_t rows, cols, ld, elem;
};

bool bad_shape(const Mat& m)
{
    if (!m.p) return false;
    if (m.ld < m.cols) return true;
    return m.rows > 0 && (m.rows - 1) > (MAX_SPAN - 1 - m.cols) / m.ld;
}

bool misaligned(const Mat& m) { return ((uintptr_t)m.p & (uintptr_t)(m.elem - 1)) != 0; }

bool overlaps(const Mat& a, const Mat& b)
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

bool same(const Mat& a, const Mat& b) { return a.p == b.p && a.ld == b.ld && a.elem == b.elem; }

// `out` against what it must not overlap; those in `may_equal` may be the same matrix.
bool clashes(const Mat& out, std::initializer_list<Mat> others, std::initializer_list<Mat> may_equal = {})
{
    for (const Mat& m : others)
        if (overlaps(out, m)) return true;
    for (const Mat& m : may_equal)
        if (!same(out, m) && overlaps(out, m)) return true;
    return false;
}

bool any_bad_shape(std::initializer_list<Mat> ms)
{
    for (const Mat& m : ms)
        if (bad_shape(m)) return true;
    return false;
}

bool any_misaligned(std::initializer_list<Mat> ms)
{
    for (const Mat& m : ms)
        if (misaligned(m)) return true;
    return false;
}

bool valid_drop(const cliff_dropout_desc* d)
{
    return !d || (d->p >= 0.0 && d->p <= 1.0 && (d->p == 0.0 || d->rng));
}

DropArgs to_args(const cliff_dropout_desc* d)
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

Mat vec(const void* p, int64_t n, int64_t elem) { return Mat{p, 1, n, n, elem}; }
Mat rng_of(const DropArgs& d) { return vec(d.rng, 2, 8); }

cliff_status check_workspace(const void* p, int64_t have, int64_t need)
{
    if (need == 0) return CLIFF_OK;
    if (!p || have < need) return CLIFF_ESCRATCH;
    return ((uintptr_t)p & 15u) ? CLIFF_EALIGN : CLIFF_OK;
}

// Widths and row counts, and the dense matrices of them (workspaces too).
bool valid_dense_sizes(int64_t M, int64_t K, int64_t N)
{
    return M >= 0 && M <= MAX_SIZE && K >= 1 && K <= MAX_SIZE && N >= 1 && N <= MAX_SIZE &&
           M * K < MAX_SPAN && M * N < MAX_SPAN && K * N < MAX_SPAN;
}

}  // namespace

extern "C" {

int64_t cliffconv_dense_workspace(int dtype, int64_t M, int64_t K, int64_t N)
{
    if (!valid_dtype(dtype) || !valid_dense_sizes(M, K, N)) return 0;
    return dense_workspace(dtype, M, K, N);
}

cliff_status cliffconv_dense(int dtype, int64_t M, int64_t K, int64_t N, const void* x,
                             int64_t ldx, const void* w, int64_t ldw, int w_out_in,
                             const void* bias, int act, const cliff_dropout_desc* drop,
                             const void* residual, int64_t ldr, void* pre, int64_t ldp, void* y,
                             int64_t ldy, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || !w || (M != 0 && (!x || !y)) || (w_out_in != 0 && w_out_in != 1) ||
        act < CLIFF_ACT_NONE || act > CLIFF_ACT_SILU || !valid_drop(drop))
        return CLIFF_EINVAL;
    if (!valid_dense_sizes(M, K, N)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mx{x, M, K, ldx, e}, mw{w, w_out_in ? N : K, w_out_in ? K : N, ldw, e},
        mb = vec(bias, N, e), mr{residual, M, N, ldr, e}, mp{pre, M, N, ldp, e}, my{y, M, N, ldy, e};
    if (any_bad_shape({mx, mw, mr, mp, my})) return CLIFF_ESHAPE;
    const DropArgs da = to_args(drop);
    if (any_misaligned({mx, mw, mb, mr, mp, my, rng_of(da)})) return CLIFF_EALIGN;
    if (clashes(my, {mx, mw, mb, mp, rng_of(da)}, {mr}) || clashes(mp, {mx, mw, mb, mr, rng_of(da)}))
        return CLIFF_EOVERLAP;
    if (M == 0) return CLIFF_OK;
    const int64_t need = dense_workspace(dtype, M, K, N);
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1), {mx, mw, mb, mr, mp, my, rng_of(da)}))
        return CLIFF_EOVERLAP;
    const DenseArgs a{M,  K,        N,   x,   ldx, w,  ldw, w_out_in, bias, act,
                      da, residual, ldr, pre, ldp, y, ldy, workspace};
    return launch_dense(dtype, a, (hipStream_t)stream);
}

int64_t cliffconv_dense_backward_workspace(int dtype, int64_t M, int64_t K, int64_t N)
{
    if (!valid_dtype(dtype) || !valid_dense_sizes(M, K, N)) return 0;
    return dense_backward_workspace(dtype, M, K, N);
}

cliff_status cliffconv_dense_backward(int dtype, int64_t M, int64_t K, int64_t N, const void* dy,
                                      int64_t lddy, const void* x, int64_t ldx, const void* w,
                                      int64_t ldw, int w_out_in, const void* pre, int64_t ldp,
                                      int act, const cliff_dropout_desc* drop, void* dx,
                                      int64_t lddx, void* dw, int64_t lddw, void* dbias,
                                      void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || !w || (M != 0 && (!dy || !x)) || (w_out_in != 0 && w_out_in != 1) ||
        act < CLIFF_ACT_NONE || act > CLIFF_ACT_SILU ||
        (M != 0 && act != CLIFF_ACT_NONE && !pre) || !valid_drop(drop))
        return CLIFF_EINVAL;
    if (act == CLIFF_ACT_NONE) pre = nullptr;
    if (!valid_dense_sizes(M, K, N)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype), wr = w_out_in ? N : K, wc = w_out_in ? K : N;
    const Mat mg{dy, M, N, lddy, e}, mx{x, M, K, ldx, e}, mw{w, wr, wc, ldw, e}, mp{pre, M, N, ldp, e},
        mdx{dx, M, K, lddx, e}, mdw{dw, wr, wc, lddw, e}, mdb = vec(dbias, N, e);
    if (any_bad_shape({mg, mx, mw, mp, mdx, mdw})) return CLIFF_ESHAPE;
    const DropArgs da = to_args(drop);
    const Mat rng = rng_of(da);
    if (any_misaligned({mg, mx, mw, mp, mdx, mdw, mdb, rng})) return CLIFF_EALIGN;
    if (clashes(mdx, {mg, mx, mw, mp, mdw, mdb, rng}) || clashes(mdw, {mg, mx, mw, mp, mdb, rng}) ||
        clashes(mdb, {mg, mx, mw, mp, rng}))
        return CLIFF_EOVERLAP;
    const int64_t need = dense_backward_workspace(dtype, M, K, N);
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1), {mg, mx, mw, mp, mdx, mdw, mdb, rng}))
        return CLIFF_EOVERLAP;
    const DenseBackwardArgs a{M,   K,  N,  dy,  lddy, x,    ldx, w,    ldw,   w_out_in, pre,
                              ldp, act, da, dx, lddx, dw, lddw, dbias, workspace};
    return launch_dense_backward(dtype, a, (hipStream_t)stream);
}

cliff_status cliffconv_layer_norm(int dtype, int64_t rows, int64_t d, const void* x, int64_t ldx,
                                  const void* weight, const void* bias, double eps, void* y,
                                  int64_t ldy, float* mean, float* rstd, void* stream)
{
    if (!valid_dtype(dtype) || (rows != 0 && (!x || !y)) || !(eps >= 0.0)) return CLIFF_EINVAL;
    if (!valid_dense_sizes(rows, d, 1)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mx{x, rows, d, ldx, e}, my{y, rows, d, ldy, e}, mw = vec(weight, d, e), mb = vec(bias, d, e),
        mm = vec(mean, rows, 4), mi = vec(rstd, rows, 4);
    if (any_bad_shape({mx, my})) return CLIFF_ESHAPE;
    if (any_misaligned({mx, my, mw, mb, mm, mi})) return CLIFF_EALIGN;
    if (clashes(my, {mw, mb, mm, mi}, {mx}) || clashes(mm, {mx, mw, mb, mi}) || clashes(mi, {mx, mw, mb}))
        return CLIFF_EOVERLAP;
    if (rows == 0) return CLIFF_OK;
    const NormArgs a{rows, d, x, ldx, weight, bias, (float)eps, y, ldy, mean, rstd};
    return launch_layer_norm(dtype, a, (hipStream_t)stream);
}

int64_t cliffconv_layer_norm_backward_workspace(int dtype, int64_t rows, int64_t d)
{
    if (!valid_dtype(dtype) || !valid_dense_sizes(rows, d, 1)) return 0;
    return layer_norm_backward_workspace(dtype, rows, d);
}

cliff_status cliffconv_layer_norm_backward(int dtype, int64_t rows, int64_t d, const void* dy,
                                           int64_t lddy, const void* x, int64_t ldx,
                                           const float* mean, const float* rstd,
                                           const void* weight, const void* dresidual, int64_t ldr,
                                           void* dx, int64_t lddx, void* dweight, void* dbias,
                                           void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || (rows != 0 && (!dy || !x || !mean || !rstd || !dx))) return CLIFF_EINVAL;
    if (!valid_dense_sizes(rows, d, 1)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mg{dy, rows, d, lddy, e}, mx{x, rows, d, ldx, e}, mr{dresidual, rows, d, ldr, e},
        mdx{dx, rows, d, lddx, e}, mw = vec(weight, d, e), mdw = vec(dweight, d, e), mdb = vec(dbias, d, e),
        mm = vec(mean, rows, 4), mi = vec(rstd, rows, 4);
    if (any_bad_shape({mg, mx, mr, mdx})) return CLIFF_ESHAPE;
    if (any_misaligned({mg, mx, mr, mdx, mw, mdw, mdb, mm, mi})) return CLIFF_EALIGN;
    if (clashes(mdx, {mx, mw, mm, mi, mdw, mdb}, {mg, mr}) ||
        clashes(mdw, {mg, mx, mr, mw, mm, mi, mdb}) || clashes(mdb, {mg, mx, mr, mw, mm, mi}))
        return CLIFF_EOVERLAP;
    const int64_t need = dweight || dbias ? layer_norm_backward_workspace(dtype, rows, d) : 0;
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1), {mg, mx, mr, mdx, mw, mdw, mdb, mm, mi}))
        return CLIFF_EOVERLAP;
    const NormBackwardArgs a{rows, d,         dy,  lddy, x,    ldx,     mean,  rstd,
                             weight, dresidual, ldr, dx,   lddx, dweight, dbias, workspace};
    return launch_layer_norm_backward(dtype, a, (hipStream_t)stream);
}

cliff_status cliffconv_dropout(int dtype, int64_t rows, int64_t d, const void* x, int64_t ldx,
                               const cliff_dropout_desc* drop, const void* residual, int64_t ldr,
                               void* y, int64_t ldy, void* stream)
{
    if (!valid_dtype(dtype) || (rows != 0 && (!x || !y)) || !drop || !valid_drop(drop)) return CLIFF_EINVAL;
    if (!valid_dense_sizes(rows, d, 1)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mx{x, rows, d, ldx, e}, mr{residual, rows, d, ldr, e}, my{y, rows, d, ldy, e};
    if (any_bad_shape({mx, mr, my})) return CLIFF_ESHAPE;
    const DropArgs da = to_args(drop);
    if (any_misaligned({mx, mr, my, rng_of(da)})) return CLIFF_EALIGN;
    if (clashes(my, {rng_of(da)}, {mx, mr})) return CLIFF_EOVERLAP;
    if (rows == 0) return CLIFF_OK;
    const DropoutArgs a{rows, d, x, ldx, da, residual, ldr, y, ldy};
    return launch_dropout(dtype, a, (hipStream_t)stream);
}

}  // extern "C"
