"""A residual feed-forward block in 8 bits (include/cliffconv_ff.h): rows quantized
to 8-bit integers and back, the dense layer of 8-bit integers for serving, the
dense layer's gradient from 8-bit checkpoints for training, and the norms after
and before a block fused with its gate and the scaled residual, with their
gradient.

Tensors, checks, plans, streams and errors are those of ``feed_forward``: rows are
the leading axes of a tensor, features its last one, and rows have one stride.
8-bit integers are int8 tensors of the same shape as the values, with float32
scales [rows, groups], contiguous: one for a row (groups = 1), or one for each
GROUP = 128 features of it (groups = ceil(features / 128)).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import paper_2507_01040_amd as _pkg

from .feed_forward import (
    ACT_NONE, CliffDropoutDesc, _Buffers, _check_act, _check_dev, _check_dropout, _check_dropout_dev,
    _check_features, _check_rows, _check_vector, _check_vector_dev, _drop_desc, _plan, _ptr, _ref,
    _row_stride, _rows_of, _shape, _stride_in_order, _type_of, _weight_order)

GROUP = 128  # CLIFF_INT8_GROUP
MAX_INT8_FEATURES = 131071  # of a dense_int8's input: its sums are 32-bit integers


class CliffBlockNormDesc(ctypes.Structure):
    _fields_ = [("after", ctypes.c_int), ("before", ctypes.c_int), ("rms", ctypes.c_int),
                ("scale", ctypes.c_double), ("eps", ctypes.c_double), ("gates", ctypes.c_int64)]


def declare(lib) -> None:
    """Argument and result types of the entry points."""
    i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    drop, norm = ctypes.POINTER(CliffDropoutDesc), ctypes.POINTER(CliffBlockNormDesc)
    mat = [vp, i64]
    lib.cliffconv_quantize.argtypes = [i32, i64, i64, *mat, i64, *mat, vp, vp]
    lib.cliffconv_dequantize.argtypes = [i32, i64, i64, *mat, vp, i64, *mat, vp]
    lib.cliffconv_dense_int8.argtypes = [i32, i64, i64, i64, *mat, vp, *mat, vp, vp, i32, *mat, *mat,
                                         vp, i64, vp]
    lib.cliffconv_dense_backward_int8.argtypes = [i32, i64, i64, i64, *mat, *mat, vp, i64, *mat, i32,
                                                  *mat, vp, i64, i32, drop, *mat, *mat, vp, vp, i64, vp]
    lib.cliffconv_block_norm.argtypes = [i32, i64, i64, norm, *mat, *mat, vp, vp, vp, vp, vp, *mat,
                                         *mat, vp, vp]
    lib.cliffconv_block_norm_backward.argtypes = [i32, i64, i64, norm, *mat, *mat, *mat, *mat, vp, vp,
                                                  vp, vp, vp, *mat, *mat, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.cliffconv_dense_int8_workspace.argtypes = [i64, i64, i64]
    lib.cliffconv_dense_backward_int8_workspace.argtypes = [i32, i64, i64, i64]
    lib.cliffconv_block_norm_backward_workspace.argtypes = [i32, i64, i64, i64]
    for name in EXPORTED:
        getattr(lib, name).restype = i64 if name.endswith("_workspace") else i32


EXPORTED = ("cliffconv_quantize", "cliffconv_dequantize", "cliffconv_dense_int8",
            "cliffconv_dense_int8_workspace", "cliffconv_dense_backward_int8",
            "cliffconv_dense_backward_int8_workspace", "cliffconv_block_norm",
            "cliffconv_block_norm_backward", "cliffconv_block_norm_backward_workspace")


# ---------------------------------------------------------------------------
# Rows in 8 bits
# ---------------------------------------------------------------------------

def _groups(d: int) -> int:
    return -(-d // GROUP)


def _check_scale(scale, rows: int, d: int, name: str, grouped: bool = True) -> int:
    """The group (0: the row) that scales [rows, groups] of d features are for."""
    want = (rows, 1), (rows, _groups(d))
    if _shape(scale) not in (want if grouped else want[:1]):
        raise ValueError("%s has shape %s, expected %s" % (
            name, _shape(scale), " or ".join(str(w) for w in (want if grouped else want[:1]))))
    return GROUP if scale.shape[1] > 1 else 0


def _check_int8_dev(q, name: str, like=None) -> None:
    import torch
    _check_dev(q, name, like, torch.int8)


def quantize_plan(x, group: Optional[int] = None, q=None, scale=None, stream=None):
    """quantize as a plan."""
    import torch
    _check_features(x, "x")
    d, rows = x.shape[-1], _rows_of(x.shape)
    if group not in (None, GROUP):
        raise ValueError("group %r is neither None nor %d" % (group, GROUP))
    shape = (rows, _groups(d) if group else 1)
    for t, want, name in ((q, x.shape, "q"), (scale, shape, "scale")):
        if t is not None:
            _check_rows(t, want, name)
    _check_dev(x, "x")
    code = _type_of(x, "x")
    b = _Buffers(x, stream)
    q = b.empty(q, tuple(x.shape), "q", torch.int8)
    scale = b.empty(scale, shape, "scale", torch.float32)
    _check_vector_dev(scale, "scale", x, torch.float32)
    args = (code, rows, d, _ptr(x), _row_stride(x, "x"), group or 0, _ptr(q), _row_stride(q, "q"),
            _ptr(scale))
    return _plan("cliffconv_quantize", args, (q, scale), (x, q, scale), stream)


def quantize(x, group: Optional[int] = None, q=None, scale=None, stream=None):
    """Rows x [..., d] in 8 bits: returns (q, scale), int8 [..., d] and float32
    [rows, groups], one scale for a row, or one for each 128 features of it where
    ``group`` is 128.  scale = max(max |x| / 127, 2^-126) of what it is for, q the
    integer nearest to x / scale (ties to even).  A group that holds an infinity
    or NaN has the scale NaN."""
    return quantize_plan(x, group, q, scale, stream)()


def dequantize_plan(q, scale, dtype=None, out=None, stream=None):
    """dequantize as a plan."""
    import torch
    _check_features(q, "q")
    d, rows = q.shape[-1], _rows_of(q.shape)
    group = _check_scale(scale, rows, d, "scale")
    if out is not None:
        _check_rows(out, q.shape, "out")
        dtype = out.dtype if dtype is None else dtype
    _check_int8_dev(q, "q")
    _check_vector_dev(scale, "scale", q, torch.float32)
    out = _Buffers(q, stream).empty(out, tuple(q.shape), "out", torch.float32 if dtype is None else dtype)
    args = (_type_of(out, "out"), rows, d, _ptr(q), _row_stride(q, "q"), _ptr(scale), group, _ptr(out),
            _row_stride(out, "out"))
    return _plan("cliffconv_dequantize", args, out, (q, scale, out), stream)


def dequantize(q, scale, dtype=None, out=None, stream=None):
    """The values q scale that 8-bit rows (quantize) stand for, of type ``dtype``
    (that of ``out``, or float32)."""
    return dequantize_plan(q, scale, dtype, out, stream)()


# ---------------------------------------------------------------------------
# Dense layer
# ---------------------------------------------------------------------------

def dense_int8_plan(x, x_scale, weight, weight_scale, bias=None, act: int = ACT_NONE, residual=None,
                    dtype=None, out=None, workspace=None, stream=None):
    """dense_int8 as a plan."""
    import torch
    _check_features(x, "x")
    K, M = x.shape[-1], _rows_of(x.shape)
    if len(_shape(weight)) != 2 or weight.shape[0] != K or weight.shape[1] < 1:
        raise ValueError("weight has shape %s, expected [%d, features out]" % (_shape(weight), K))
    if K > MAX_INT8_FEATURES:
        raise ValueError("x has %d features, expected at most %d" % (K, MAX_INT8_FEATURES))
    N = weight.shape[1]
    shape = tuple(x.shape[:-1]) + (N,)
    _check_scale(x_scale, M, K, "x_scale", grouped=False)
    _check_scale(weight_scale, N, K, "weight_scale", grouped=False)
    _check_vector(bias, N, "bias")
    _check_act(act)
    for t, name in ((residual, "residual"), (out, "out")):
        if t is not None:
            _check_rows(t, shape, name)
    _check_int8_dev(x, "x")
    _check_int8_dev(weight, "weight", x)
    _check_vector_dev(x_scale, "x_scale", x, torch.float32)
    _check_vector_dev(weight_scale, "weight_scale", x, torch.float32)
    ldw = _stride_in_order(weight, 1)
    if ldw is None:
        raise ValueError("weight is not the transposed view of a stored [features out, features in] "
                         "(shape %s, strides %s)" % (tuple(weight.shape), tuple(weight.stride())))
    if dtype is None:
        like = out if out is not None else residual if residual is not None else bias
        dtype = like.dtype if like is not None else torch.bfloat16
    b = _Buffers(x, stream)
    out = b.empty(out, shape, "out", dtype)
    code = _type_of(out, "out")
    _check_vector_dev(bias, "bias", x, dtype)
    if residual is not None:
        _check_dev(residual, "residual", x, dtype)
    ws, ws_bytes = b.workspace(workspace, _pkg.load().cliffconv_dense_int8_workspace(M, K, N))
    args = (code, M, K, N, _ptr(x), _row_stride(x, "x"), _ptr(x_scale), _ptr(weight), ldw,
            _ptr(weight_scale), _ptr(bias), act, _ptr(residual),
            _row_stride(residual, "residual") if residual is not None else 0, _ptr(out),
            _row_stride(out, "out"), _ptr(ws), ws_bytes)
    return _plan("cliffconv_dense_int8", args, out,
                 (x, x_scale, weight, weight_scale, bias, residual, out, ws), stream)


def dense_int8(x, x_scale, weight, weight_scale, bias=None, act: int = ACT_NONE, residual=None,
               dtype=None, out=None, workspace=None, stream=None):
    """Dense layer residual + f(x_scale weight_scale (x weight) + bias) of 8-bit
    integers: x int8 [..., K] with x_scale [rows, 1], as ``quantize`` gives them for
    the input, and weight int8 [K, N] with weight_scale [N, 1], the transposed view
    and the scales that it gives for the weight stored [N, K].  The sums are exact; K
    is at most 131071.  The output [..., N], bias and residual have the type
    ``dtype`` (that of out, residual or bias if one is given, else bfloat16)."""
    return dense_int8_plan(x, x_scale, weight, weight_scale, bias, act, residual, dtype, out, workspace,
                           stream)()


def dense_backward_int8_plan(dy, x, x_scale, weight, pre=None, pre_scale=None, act: int = ACT_NONE,
                             dropout=None, bias: bool = True, dx=None, dweight=None, dbias=None,
                             workspace=None, stream=None):
    """dense_backward_int8 as a plan."""
    import torch
    _check_features(x, "x")
    K, M = x.shape[-1], _rows_of(x.shape)
    if len(_shape(weight)) != 2 or weight.shape[0] != K or weight.shape[1] < 1:
        raise ValueError("weight has shape %s, expected [%d, features out]" % (_shape(weight), K))
    N = weight.shape[1]
    _check_rows(dy, tuple(x.shape[:-1]) + (N,), "dy")
    x_group = _check_scale(x_scale, M, K, "x_scale")
    _check_act(act)
    _check_dropout(dropout)
    pre_group = 0
    if act != ACT_NONE:
        if pre is None or pre_scale is None:
            raise ValueError("an activation's gradient needs the pre-activations and their scales")
        _check_rows(pre, dy.shape, "pre")
        pre_group = _check_scale(pre_scale, M, N, "pre_scale")
    else:
        pre = pre_scale = None
    for t, like, name in ((dx, x, "dx"), (dweight, weight, "dweight")):
        if t is not None and t is not False:
            _check_rows(t, like.shape, name)
    if dbias is not None:
        _check_vector(dbias, N, "dbias")
    _check_dev(dy, "dy")
    code = _type_of(dy, "dy")
    _check_int8_dev(x, "x", dy)
    _check_vector_dev(x_scale, "x_scale", dy, torch.float32)
    _check_dev(weight, "weight", dy)
    if pre is not None:
        _check_int8_dev(pre, "pre", dy)
        _check_vector_dev(pre_scale, "pre_scale", dy, torch.float32)
    _check_dropout_dev(dropout, dy)
    order, ldw = _weight_order(weight, like=None if dweight is False else dweight)
    b = _Buffers(dy, stream)
    dx = None if dx is False else b.empty(dx, tuple(x.shape), "dx")
    if dweight is False:
        dweight = None
    elif dweight is None:  # in the order of the weight
        dweight = b.empty(None, (N, K), "dweight").t() if order else b.empty(None, (K, N), "dweight")
    else:
        b.empty(dweight, (K, N), "dweight")
    lddw = _stride_in_order(dweight, order) if dweight is not None else N
    if bias:
        dbias = b.empty(dbias, (N,), "dbias")
        _check_vector_dev(dbias, "dbias", dy)
    else:
        dbias = None
    ws, ws_bytes = b.workspace(workspace,
                               _pkg.load().cliffconv_dense_backward_int8_workspace(code, M, K, N))
    desc = _drop_desc(dropout)
    args = (code, M, K, N, _ptr(dy), _row_stride(dy, "dy"), _ptr(x), _row_stride(x, "x"), _ptr(x_scale),
            x_group, _ptr(weight), ldw, order, _ptr(pre),
            _row_stride(pre, "pre") if pre is not None else 0, _ptr(pre_scale), pre_group, act,
            _ref(desc), _ptr(dx), _row_stride(dx, "dx") if dx is not None else 0, _ptr(dweight), lddw,
            _ptr(dbias), _ptr(ws), ws_bytes)
    outs = tuple(t for t, want in ((dx, dx is not None), (dweight, dweight is not None),
                                   (dbias, bool(bias))) if want)
    return _plan("cliffconv_dense_backward_int8", args, outs,
                 (dy, x, x_scale, weight, pre, pre_scale, dropout, dx, dweight, dbias, ws, desc), stream)


def dense_backward_int8(dy, x, x_scale, weight, pre=None, pre_scale=None, act: int = ACT_NONE,
                        dropout=None, bias: bool = True, dx=None, dweight=None, dbias=None,
                        workspace=None, stream=None):
    """dense_backward from checkpoints in 8 bits: x int8 [..., K] and pre int8
    [..., N] with their scales, as ``quantize`` gave them (group None or 128, each
    its own) for the forward call's input and pre-activations.  The rest is as
    there."""
    return dense_backward_int8_plan(dy, x, x_scale, weight, pre, pre_scale, act, dropout, bias, dx,
                                    dweight, dbias, workspace, stream)()


# ---------------------------------------------------------------------------
# The norms around a block
# ---------------------------------------------------------------------------

class BlockNormGradients(NamedTuple):
    """What block_norm_backward returns; None where there is no such input."""
    dx: object
    dresidual: object
    dgate: object = None
    dweight: object = None
    dbias: object = None
    dnext_weight: object = None
    dnext_bias: object = None


def _check_gate(gate, rows: int, d: int) -> int:
    """The number of a gate's rows: [d], or [gates, d] with gates a divisor of the rows."""
    if gate is None:
        return 1
    shape = _shape(gate)
    if shape == (d,):
        return 1
    if len(shape) != 2 or shape[1] != d or shape[0] < 1 or rows % shape[0]:
        raise ValueError("gate has shape %s, expected (%d,) or (a divisor of %d rows, %d)"
                         % (shape, d, rows, d))
    return shape[0]


def _norm_desc(after, before, rms, scale, eps, gates) -> CliffBlockNormDesc:
    scale, eps = float(scale), float(eps)
    if not abs(scale) < 3.4e38:
        raise ValueError("scale %r is not a finite float32" % (scale,))
    if not eps >= 0.0:
        raise ValueError("eps %r is negative" % (eps,))
    if not after and not before:
        raise ValueError("neither norm is asked for")
    return CliffBlockNormDesc(int(bool(after)), int(bool(before)), int(bool(rms)), scale, eps, gates)


def _check_norm_vectors(vectors, wanted: bool, which: str, d: int) -> None:
    for t, name in vectors:
        if t is not None and not wanted:
            raise ValueError("%s is given, but not the norm %s" % (name, which))
        _check_vector(t, d, name)


def block_norm_plan(x, residual, gate=None, scale: float = 1.0, weight=None, bias=None,
                    next_weight=None, next_bias=None, after: bool = True, before: bool = True,
                    rms: bool = False, eps: float = 1e-5, out=None, normed=None, stats=None,
                    stream=None):
    """block_norm as a plan."""
    import torch
    _check_features(x, "x")
    d, rows = x.shape[-1], _rows_of(x.shape)
    _check_rows(residual, x.shape, "residual")
    gates = _check_gate(gate, rows, d)
    _check_norm_vectors(((weight, "weight"), (bias, "bias")), after, "after the block", d)
    _check_norm_vectors(((next_weight, "next_weight"), (next_bias, "next_bias")), before,
                        "before the next block", d)
    if normed is not None and not before:
        raise ValueError("normed is given, but not the norm before the next block")
    for t, shape, name in ((out, x.shape, "out"), (normed, x.shape, "normed"), (stats, (4, rows), "stats")):
        if t is not None:
            _check_rows(t, shape, name)
    desc = _norm_desc(after, before, rms, scale, eps, gates)
    _check_dev(x, "x")
    code = _type_of(x, "x")
    _check_dev(residual, "residual", x)
    for t, name in ((gate, "gate"), (weight, "weight"), (bias, "bias"), (next_weight, "next_weight"),
                    (next_bias, "next_bias")):
        _check_vector_dev(t, name, x)
    b = _Buffers(x, stream)
    out = b.empty(out, tuple(x.shape), "out")
    normed = b.empty(normed, tuple(x.shape), "normed") if before else None
    stats = b.empty(stats, (4, rows), "stats", torch.float32)
    _check_vector_dev(stats, "stats", x, torch.float32)
    args = (code, rows, d, _ref(desc), _ptr(x), _row_stride(x, "x"), _ptr(residual),
            _row_stride(residual, "residual"), _ptr(gate), _ptr(weight), _ptr(bias), _ptr(next_weight),
            _ptr(next_bias), _ptr(out), _row_stride(out, "out"), _ptr(normed),
            _row_stride(normed, "normed") if before else 0, _ptr(stats))
    return _plan("cliffconv_block_norm", args, (out, normed, stats) if before else (out, stats),
                 (x, residual, gate, weight, bias, next_weight, next_bias, out, normed, stats, desc),
                 stream)


def block_norm(x, residual, gate=None, scale: float = 1.0, weight=None, bias=None, next_weight=None,
               next_bias=None, after: bool = True, before: bool = True, rms: bool = False,
               eps: float = 1e-5, out=None, normed=None, stats=None, stream=None):
    """What stands between two blocks, of x [..., d] that a block gives and the
    residual rows [..., d] that went past it:

        out = scale residual + gate n(x; weight, bias)
        normed = n(out; next_weight, next_bias)

    n is layer norm, or with ``rms`` the same without mean.  Without ``after`` x
    itself takes the place of its norm, without ``before`` there is no normed.
    ``gate`` is [d], or [gates, d] where each is for rows / gates neighbouring
    rows; vectors are [d].  Returns (out, normed, stats), or (out, stats) without
    ``before``: stats float32 [4, rows] holds mean and rstd of x and of out, for the
    gradient (those of a norm that is not taken are not written).  ``out`` and
    ``normed`` may each be x or residual."""
    return block_norm_plan(x, residual, gate, scale, weight, bias, next_weight, next_bias, after, before,
                           rms, eps, out, normed, stats, stream)()


def block_norm_backward_plan(dout, dnormed, x, out, stats, gate=None, scale: float = 1.0, weight=None,
                             bias=None, next_weight=None, next_bias=None, after: bool = True,
                             rms: bool = False, params: bool = True, dx=None, dresidual=None,
                             dgate=None, dweight=None, dbias=None, dnext_weight=None, dnext_bias=None,
                             workspace=None, stream=None):
    """block_norm_backward as a plan."""
    import torch
    like = dnormed if dnormed is not None else dout
    if like is None:
        raise ValueError("neither dout nor dnormed is given")
    before = dnormed is not None
    _check_features(like, "dout" if dnormed is None else "dnormed")
    shape, d, rows = tuple(like.shape), like.shape[-1], _rows_of(like.shape)
    gates = _check_gate(gate, rows, d)
    reads_x = after or (params and gate is not None)
    for t, wanted, name in ((dout, False, "dout"), (x, reads_x, "x"), (out, before, "out"),
                            (dx, False, "dx"), (dresidual, False, "dresidual")):
        if t is not None or wanted:
            _check_rows(t, shape, name)
    _check_rows(stats, (4, rows), "stats")
    _check_norm_vectors(((weight, "weight"), (bias, "bias"), (dweight, "dweight"), (dbias, "dbias")),
                        after, "after the block", d)
    _check_norm_vectors(((next_weight, "next_weight"), (next_bias, "next_bias"),
                         (dnext_weight, "dnext_weight"), (dnext_bias, "dnext_bias")), before,
                        "before the next block", d)
    desc = _norm_desc(after, before, rms, scale, 0.0, gates)
    _check_dev(like, "dout" if dnormed is None else "dnormed")
    code = _type_of(like, "dout")
    for t, name in ((dout, "dout"), (x if reads_x else None, "x"), (out if before else None, "out")):
        if t is not None:
            _check_dev(t, name, like)
    _check_vector_dev(stats, "stats", like, torch.float32)
    for t, name in ((gate, "gate"), (weight, "weight"), (bias, "bias"), (next_weight, "next_weight"),
                    (next_bias, "next_bias")):
        _check_vector_dev(t, name, like)
    b = _Buffers(like, stream)
    dx, dresidual = b.empty(dx, shape, "dx"), b.empty(dresidual, shape, "dresidual")

    def sums(of, given, name):
        if of is None or not params:
            if given is not None:
                raise ValueError("%s is given, but not wanted" % name)
            return None
        if given is not None:
            _check_rows(given, of.shape, name)
        given = b.empty(given, tuple(of.shape), name)
        _check_vector_dev(given, name, like)
        return given

    dgate = sums(gate, dgate, "dgate")
    dweight, dbias = sums(weight, dweight, "dweight"), sums(bias, dbias, "dbias")
    dnext_weight = sums(next_weight, dnext_weight, "dnext_weight")
    dnext_bias = sums(next_bias, dnext_bias, "dnext_bias")
    need = _pkg.load().cliffconv_block_norm_backward_workspace(code, rows, d, gates if gate is not None else 0)
    ws, ws_bytes = b.workspace(workspace, need)
    args = (code, rows, d, _ref(desc), _ptr(dout), _row_stride(dout, "dout") if dout is not None else 0,
            _ptr(dnormed), _row_stride(dnormed, "dnormed") if before else 0,
            _ptr(x) if reads_x else None, _row_stride(x, "x") if reads_x else 0,
            _ptr(out) if before else None, _row_stride(out, "out") if before else 0, _ptr(stats),
            _ptr(gate), _ptr(weight), _ptr(bias), _ptr(next_weight), _ptr(dx), _row_stride(dx, "dx"),
            _ptr(dresidual), _row_stride(dresidual, "dresidual"), _ptr(dgate), _ptr(dweight), _ptr(dbias),
            _ptr(dnext_weight), _ptr(dnext_bias), _ptr(ws), ws_bytes)
    return _plan("cliffconv_block_norm_backward", args,
                 BlockNormGradients(dx, dresidual, dgate, dweight, dbias, dnext_weight, dnext_bias),
                 (like, dout, x, out, stats, gate, weight, bias, next_weight, next_bias, dx, dresidual,
                  dgate, dweight, dbias, dnext_weight, dnext_bias, ws, desc), stream)


def block_norm_backward(dout, dnormed, x, out, stats, gate=None, scale: float = 1.0, weight=None,
                        bias=None, next_weight=None, next_bias=None, after: bool = True,
                        rms: bool = False, params: bool = True, dx=None, dresidual=None, dgate=None,
                        dweight=None, dbias=None, dnext_weight=None, dnext_bias=None, workspace=None,
                        stream=None):
    """Gradient of block_norm for the gradients of its outputs, dout (what out gets
    past the next norm, or None) and dnormed (None for a call without ``before``):
    returns BlockNormGradients (dx, dresidual, dgate, dweight, dbias, dnext_weight,
    dnext_bias).  x, out, stats, the gate and the vectors are those of the forward
    call; each gate and vector that is given gets its gradient, of its shape, and
    none does where ``params`` is False.  x may be None without ``after`` if no
    gate's gradient is wanted, out without ``before``.  ``dx`` and ``dresidual`` may
    each be dout or dnormed."""
    return block_norm_backward_plan(dout, dnormed, x, out, stats, gate, scale, weight, bias, next_weight,
                                    next_bias, after, rms, params, dx, dresidual, dgate, dweight, dbias,
                                    dnext_weight, dnext_bias, workspace, stream)()
