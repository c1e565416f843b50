// C ABI of the 8-bit operators and the block norm (cliffconv_ff.h): argument
// checks and dispatch.  No device memory is allocated here; every call only
// enqueues kernels on the caller's stream.
#include "cliffconv_ff.h"
#include "ff_common.hpp"

using namespace cliff;

namespace {

constexpr int64_t GROUP = CLIFF_INT8_GROUP;
constexpr int64_t MAX_INT8_K = 131071;  // (-128)^2 times it is below 2^31

bool valid_group(int64_t group) { return group == 0 || group == GROUP; }
int64_t groups_of(int64_t group, int64_t d) { return group ? (d + group - 1) / group : 1; }

// scales [rows, groups]
Mat scales(const void* p, int64_t rows, int64_t groups)
{
    return rows ? vec(p, rows * groups, 4) : Mat{nullptr, 0, 1, 1, 4};
}

bool valid_block_norm(const cliff_block_norm_desc* d)
{
    return d && (d->after || d->before) && isfinite((float)d->scale) && d->eps >= 0.0;
}

}  // namespace

extern "C" {

cliff_status cliffconv_quantize(int dtype, int64_t rows, int64_t d, const void* x, int64_t ldx, int64_t group,
                                int8_t* q, int64_t ldq, float* scale, void* stream)
{
    if (!valid_dtype(dtype) || (rows != 0 && (!x || !q || !scale)) || !valid_group(group)) return CLIFF_EINVAL;
    if (!valid_dense_sizes(rows, d, 1)) return CLIFF_ESHAPE;
    const int64_t groups = groups_of(group, d);
    const Mat mx{x, rows, d, ldx, size_of(dtype)}, mq{q, rows, d, ldq, 1}, ms = scales(scale, rows, groups);
    if (any_bad_shape({mx, mq})) return CLIFF_ESHAPE;
    if (any_misaligned({mx, ms})) return CLIFF_EALIGN;
    if (clashes(mq, {mx, ms}) || clashes(ms, {mx})) return CLIFF_EOVERLAP;
    if (rows == 0) return CLIFF_OK;
    return launch_quantize(dtype, QuantizeArgs{rows, d, groups, x, ldx, q, ldq, scale}, (hipStream_t)stream);
}

cliff_status cliffconv_dequantize(int dtype, int64_t rows, int64_t d, const int8_t* q, int64_t ldq, const float* scale,
                                  int64_t group, void* y, int64_t ldy, void* stream)
{
    if (!valid_dtype(dtype) || (rows != 0 && (!y || !q || !scale)) || !valid_group(group)) return CLIFF_EINVAL;
    if (!valid_dense_sizes(rows, d, 1)) return CLIFF_ESHAPE;
    const int64_t groups = groups_of(group, d);
    const Mat my{y, rows, d, ldy, size_of(dtype)}, mq{q, rows, d, ldq, 1}, ms = scales(scale, rows, groups);
    if (any_bad_shape({my, mq})) return CLIFF_ESHAPE;
    if (any_misaligned({my, ms})) return CLIFF_EALIGN;
    if (clashes(my, {mq, ms})) return CLIFF_EOVERLAP;
    if (rows == 0) return CLIFF_OK;
    return launch_dequantize(dtype, DequantizeArgs{rows, d, groups, q, ldq, scale, y, ldy}, (hipStream_t)stream);
}

int64_t cliffconv_dense_int8_workspace(int64_t M, int64_t K, int64_t N)
{
    if (!valid_dense_sizes(M, K, N) || K > MAX_INT8_K) return 0;
    return dense_int8_workspace(M, K, N);
}

cliff_status cliffconv_dense_int8(int dtype, int64_t M, int64_t K, int64_t N, const int8_t* x, int64_t ldx,
                                  const float* x_scale, const int8_t* w, int64_t ldw, const float* w_scale,
                                  const void* bias, int act, const void* residual, int64_t ldr, void* y, int64_t ldy,
                                  void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || !w || !w_scale || (M != 0 && (!x || !x_scale || !y)) || act < CLIFF_ACT_NONE ||
        act > CLIFF_ACT_SILU)
        return CLIFF_EINVAL;
    if (!valid_dense_sizes(M, K, N) || K > MAX_INT8_K) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mx{x, M, K, ldx, 1}, mw{w, N, K, ldw, 1}, mr{residual, M, N, ldr, e}, my{y, M, N, ldy, e},
        mxs = scales(x_scale, M, 1), mws = scales(w_scale, N, 1), mb = vec(bias, N, e);
    if (any_bad_shape({mx, mw, mr, my})) return CLIFF_ESHAPE;
    if (any_misaligned({mxs, mws, mb, mr, my})) return CLIFF_EALIGN;
    if (clashes(my, {mx, mw, mxs, mws, mb}, {mr})) return CLIFF_EOVERLAP;
    if (M == 0) return CLIFF_OK;
    const int64_t need = dense_int8_workspace(M, K, N);
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1), {mx, mw, mxs, mws, mb, mr, my})) return CLIFF_EOVERLAP;
    const DenseInt8Args a{M, K, N, x, ldx, x_scale, w, ldw, w_scale, bias, act, residual, ldr, y, ldy, workspace};
    return launch_dense_int8(dtype, a, (hipStream_t)stream);
}

int64_t cliffconv_dense_backward_int8_workspace(int dtype, int64_t M, int64_t K, int64_t N)
{
    if (!valid_dtype(dtype) || !valid_dense_sizes(M, K, N)) return 0;
    return dense_backward_int8_workspace(dtype, M, K, N);
}

cliff_status cliffconv_dense_backward_int8(
    int dtype, int64_t M, int64_t K, int64_t N, const void* dy, int64_t lddy, const int8_t* x, int64_t ldx,
    const float* x_scale, int64_t x_group, const void* w, int64_t ldw, int w_out_in, const int8_t* pre, int64_t ldp,
    const float* pre_scale, int64_t pre_group, int act, const cliff_dropout_desc* drop, void* dx, int64_t lddx,
    void* dw, int64_t lddw, void* dbias, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || !w || (M != 0 && (!dy || !x || !x_scale)) || (w_out_in != 0 && w_out_in != 1) ||
        act < CLIFF_ACT_NONE || act > CLIFF_ACT_SILU || (M != 0 && act != CLIFF_ACT_NONE && (!pre || !pre_scale)) ||
        !valid_drop(drop) || !valid_group(x_group) || !valid_group(pre_group))
        return CLIFF_EINVAL;
    if (act == CLIFF_ACT_NONE) pre = nullptr, pre_scale = nullptr;
    if (!valid_dense_sizes(M, K, N)) return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype), wr = w_out_in ? N : K, wc = w_out_in ? K : N;
    const int64_t xg = groups_of(x_group, K), pg = groups_of(pre_group, N);
    const Mat mg{dy, M, N, lddy, e}, mx{x, M, K, ldx, 1}, mw{w, wr, wc, ldw, e}, mp{pre, M, N, ldp, 1},
        mxs = scales(x_scale, M, xg), mps = scales(pre_scale, M, pg), mdx{dx, M, K, lddx, e}, mdw{dw, wr, wc, lddw, e},
        mdb = vec(dbias, N, e);
    if (any_bad_shape({mg, mx, mw, mp, mdx, mdw})) return CLIFF_ESHAPE;
    const DropArgs da = to_args(drop);
    const Mat rng = rng_of(da);
    if (any_misaligned({mg, mxs, mps, mw, mdx, mdw, mdb, rng})) return CLIFF_EALIGN;
    if (clashes(mdx, {mg, mx, mxs, mw, mp, mps, mdw, mdb, rng}) || clashes(mdw, {mg, mx, mxs, mw, mp, mps, mdb, rng}) ||
        clashes(mdb, {mg, mx, mxs, mw, mp, mps, rng}))
        return CLIFF_EOVERLAP;
    const int64_t need = dense_backward_int8_workspace(dtype, M, K, N);
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1), {mg, mx, mxs, mw, mp, mps, mdx, mdw, mdb, rng}))
        return CLIFF_EOVERLAP;
    const DenseBackwardInt8Args a{{M,   K,  N,  dy,  lddy, x,    ldx, w,    ldw,   w_out_in, pre,
                                   ldp, act, da, dx, lddx, dw, lddw, dbias, workspace},
                                  x_scale, xg, pre_scale, pg};
    return launch_dense_backward_int8(dtype, a, (hipStream_t)stream);
}

cliff_status cliffconv_block_norm(int dtype, int64_t rows, int64_t d, const cliff_block_norm_desc* desc, const void* x,
                                  int64_t ldx, const void* residual, int64_t ldr, const void* gate, const void* weight,
                                  const void* bias, const void* next_weight, const void* next_bias, void* out,
                                  int64_t ldo, void* normed, int64_t ldn, float* stats, void* stream)
{
    if (!valid_dtype(dtype) || !valid_block_norm(desc) || (rows != 0 && (!x || !residual || !out)) ||
        (rows != 0 && desc->before && !normed) || (!desc->after && (weight || bias)) ||
        (!desc->before && (normed || next_weight || next_bias)))
        return CLIFF_EINVAL;
    const int64_t gates = gate ? desc->gates : 0;
    if (!valid_dense_sizes(rows, d, 1) || (gate && (gates < 1 || gates > MAX_SIZE || rows % gates || gates * d >= MAX_SPAN)))
        return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mx{x, rows, d, ldx, e}, mr{residual, rows, d, ldr, e}, mo{out, rows, d, ldo, e}, mn{normed, rows, d, ldn, e},
        mg{gate, gates, d, d, e}, mw = vec(weight, d, e), mb = vec(bias, d, e), mnw = vec(next_weight, d, e),
        mnb = vec(next_bias, d, e), ms = scales(stats, rows, 4);
    if (any_bad_shape({mx, mr, mo, mn})) return CLIFF_ESHAPE;
    if (any_misaligned({mx, mr, mo, mn, mg, mw, mb, mnw, mnb, ms})) return CLIFF_EALIGN;
    if (clashes(mo, {mn, mg, mw, mb, mnw, mnb, ms}, {mx, mr}) || clashes(mn, {mg, mw, mb, mnw, mnb, ms}, {mx, mr}) ||
        clashes(ms, {mx, mr, mg, mw, mb, mnw, mnb}))
        return CLIFF_EOVERLAP;
    if (rows == 0) return CLIFF_OK;
    const BlockNormArgs a{rows, d, x, ldx, residual, ldr, gate, gates, (float)desc->scale, (float)desc->eps,
                          desc->after != 0, desc->before != 0, desc->rms != 0, weight, bias, next_weight, next_bias,
                          out, ldo, normed, ldn, stats};
    return launch_block_norm(dtype, a, (hipStream_t)stream);
}

int64_t cliffconv_block_norm_backward_workspace(int dtype, int64_t rows, int64_t d, int64_t gates)
{
    if (!valid_dtype(dtype) || !valid_dense_sizes(rows, d, 1) || gates < 0 || gates > MAX_SIZE) return 0;
    return block_norm_backward_workspace(dtype, rows, d, gates);
}

cliff_status cliffconv_block_norm_backward(
    int dtype, int64_t rows, int64_t d, const cliff_block_norm_desc* desc, const void* dout, int64_t lddo,
    const void* dnormed, int64_t lddn, const void* x, int64_t ldx, const void* out, int64_t ldo, const float* stats,
    const void* gate, const void* weight, const void* bias, const void* next_weight, void* dx, int64_t lddx,
    void* dresidual, int64_t lddr, void* dgate, void* dweight, void* dbias, void* dnext_weight, void* dnext_bias,
    void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!valid_dtype(dtype) || !valid_block_norm(desc) || (!desc->after && (weight || bias || dweight || dbias)) ||
        (!desc->before && (dnormed || next_weight || dnext_weight || dnext_bias)) || (!gate && dgate))
        return CLIFF_EINVAL;
    const bool reads_x = desc->after || dgate;
    if (rows != 0 && (!dx || !dresidual || !stats || (reads_x && !x) || (desc->before ? !dnormed || !out : !dout)))
        return CLIFF_EINVAL;
    if (!reads_x) x = nullptr;
    if (!desc->before) out = nullptr;
    const int64_t gates = gate ? desc->gates : 0;
    if (!valid_dense_sizes(rows, d, 1) || (gate && (gates < 1 || gates > MAX_SIZE || rows % gates || gates * d >= MAX_SPAN)))
        return CLIFF_ESHAPE;
    const int64_t e = size_of(dtype);
    const Mat mdo{dout, rows, d, lddo, e}, mdn{dnormed, rows, d, lddn, e}, mx{x, rows, d, ldx, e}, mo{out, rows, d, ldo, e},
        mg{gate, gates, d, d, e}, mw = vec(weight, d, e), mb = vec(bias, d, e), mnw = vec(next_weight, d, e),
        ms = scales(stats, rows, 4), mdx{dx, rows, d, lddx, e}, mdr{dresidual, rows, d, lddr, e},
        mdg{dgate, gates, d, d, e}, mdw = vec(dweight, d, e), mdb = vec(dbias, d, e), mdnw = vec(dnext_weight, d, e),
        mdnb = vec(dnext_bias, d, e);
    if (any_bad_shape({mdo, mdn, mx, mo, mdx, mdr})) return CLIFF_ESHAPE;
    if (any_misaligned({mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdx, mdr, mdg, mdw, mdb, mdnw, mdnb})) return CLIFF_EALIGN;
    if (clashes(mdx, {mx, mo, mg, mw, mb, mnw, ms, mdr, mdg, mdw, mdb, mdnw, mdnb}, {mdo, mdn}) ||
        clashes(mdr, {mx, mo, mg, mw, mb, mnw, ms, mdg, mdw, mdb, mdnw, mdnb}, {mdo, mdn}) ||
        clashes(mdg, {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdw, mdb, mdnw, mdnb}) ||
        clashes(mdw, {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdb, mdnw, mdnb}) ||
        clashes(mdb, {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdnw, mdnb}) ||
        clashes(mdnw, {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdnb}) ||
        clashes(mdnb, {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms}))
        return CLIFF_EOVERLAP;
    const int64_t need = block_norm_backward_workspace(dtype, rows, d, gates);
    const cliff_status s = check_workspace(workspace, workspace_bytes, need);
    if (s != CLIFF_OK) return s;
    if (clashes(vec(need ? workspace : nullptr, need, 1),
                {mdo, mdn, mx, mo, mg, mw, mb, mnw, ms, mdx, mdr, mdg, mdw, mdb, mdnw, mdnb}))
        return CLIFF_EOVERLAP;
    const BlockNormBackwardArgs a{rows, d, dout, lddo, dnormed, lddn, x, ldx, out, ldo, stats, gate, gates,
                                  (float)desc->scale, desc->after != 0, desc->rms != 0, weight, bias, next_weight, dx,
                                  lddx, dresidual, lddr, dgate, dweight, dbias, dnext_weight, dnext_bias, workspace};
    return launch_block_norm_backward(dtype, a, (hipStream_t)stream);
}

}  // extern "C"
