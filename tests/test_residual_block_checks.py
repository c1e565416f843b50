"""Refusals of the 8-bit operators and the block norm, on the CPU: the binding's checks
of shape-only ("meta") tensors, what it passes to the library, and the C ABI's checks of
addresses that are never dereferenced (each case carries a defect that the library must
report before any device work)."""
import ctypes

import pytest
import torch

import paper_2507_01040_amd as P
from paper_2507_01040_amd import feed_forward as F
from paper_2507_01040_amd import residual_block as R
from test_feed_forward_arguments import _Stream, library as ff_library, streams  # noqa: F401
from test_feed_forward_checks import FAKE, MB, _call, _drop, _raises, lib, m, no_library  # noqa: F401

I8 = torch.int8


def test_quantize_checks(no_library):  # noqa: F811
    _raises(lambda: P.quantize(m(6, 300)), "x must be a GPU tensor")
    _raises(lambda: P.quantize(m(6, 0)), "x has shape")
    _raises(lambda: P.quantize(m(6, 300), group=64), "group 64 is neither")
    _raises(lambda: P.quantize(m(6, 300), q=m(6, 299, dtype=I8)), "q has shape")
    _raises(lambda: P.quantize(m(6, 300), scale=m(6, 3)), "scale has shape")
    _raises(lambda: P.quantize(m(6, 300), group=128, scale=m(6, 1)), "scale has shape")
    _raises(lambda: P.quantize(m(6, 300), group=128, scale=m(6)), "scale has shape")
    _raises(lambda: P.dequantize(m(6, 300, dtype=I8), m(6, 2)), "scale has shape")
    _raises(lambda: P.dequantize(m(6, 300, dtype=I8), m(5, 1)), "scale has shape")
    _raises(lambda: P.dequantize(m(6, 300, dtype=I8), m(6, 3)), "q must be a GPU tensor")
    _raises(lambda: P.dequantize(m(6, 300, dtype=I8), m(6, 3), out=m(6, 30)), "out has shape")


def test_dense_int8_checks(no_library):  # noqa: F811
    ok = dict(x=m(6, 8, dtype=I8), x_scale=m(6, 1), weight=m(8, 5, dtype=I8), weight_scale=m(5, 1))
    _raises(lambda: P.dense_int8(**ok), "x must be a GPU tensor")
    _raises(lambda: P.dense_int8(**{**ok, "x_scale": m(6)}), "x_scale has shape")
    _raises(lambda: P.dense_int8(**{**ok, "weight": m(5, 8, dtype=I8)}), "weight has shape")
    _raises(lambda: P.dense_int8(**{**ok, "weight_scale": m(8, 1)}), "weight_scale has shape")
    _raises(lambda: P.dense_int8(**ok, bias=m(6)), "bias has shape")
    _raises(lambda: P.dense_int8(**ok, act=7), "unknown activation")
    _raises(lambda: P.dense_int8(**ok, residual=m(6, 8)), "residual has shape")
    _raises(lambda: P.dense_int8(**ok, out=m(5, 6)), "out has shape")
    # scales of 128 features are for checkpoints
    wide = dict(x=m(6, 300, dtype=I8), weight=m(300, 5, dtype=I8), weight_scale=m(5, 1))
    _raises(lambda: P.dense_int8(x_scale=m(6, 3), **wide), "x_scale has shape")
    long = dict(x=m(2, 131072, dtype=I8), x_scale=m(2, 1), weight=m(131072, 5, dtype=I8), weight_scale=m(5, 1))
    _raises(lambda: P.dense_int8(**long), "at most 131071")


def test_dense_backward_int8_checks(no_library):  # noqa: F811
    ok = dict(dy=m(6, 5), x=m(6, 300, dtype=I8), x_scale=m(6, 3), weight=m(300, 5))
    call = P.dense_backward_int8
    _raises(lambda: call(**ok), "dy must be a GPU tensor")
    _raises(lambda: call(**{**ok, "dy": m(6, 6)}), "dy has shape")
    _raises(lambda: call(**{**ok, "x_scale": m(6, 2)}), "x_scale has shape")
    _raises(lambda: call(**ok, act=P.ACT_GELU), "needs the pre-activations and their scales")
    _raises(lambda: call(**ok, act=P.ACT_GELU, pre=m(6, 5, dtype=I8)), "needs the pre-activations and their scales")
    _raises(lambda: call(**ok, act=P.ACT_GELU, pre=m(6, 5, dtype=I8), pre_scale=m(6, 5)), "pre_scale has shape")
    _raises(lambda: call(**ok, act=P.ACT_GELU, pre=m(5, 5, dtype=I8), pre_scale=m(6, 1)), "pre has shape")
    _raises(lambda: call(**ok, dropout=(2.0, m(2))), "probability")
    _raises(lambda: call(**ok, dx=m(6, 5)), "dx has shape")
    _raises(lambda: call(**ok, dweight=m(5, 300)), "dweight has shape")
    _raises(lambda: call(**ok, dbias=m(300)), "dbias has shape")


def test_block_norm_checks(no_library):  # noqa: F811
    ok, call = dict(x=m(6, 8), residual=m(6, 8)), P.block_norm
    _raises(lambda: call(**ok), "x must be a GPU tensor")
    _raises(lambda: call(m(6, 8), m(6, 7)), "residual has shape")
    for gate in (m(7), m(4, 8), m(0, 8), m(6, 7), m(2, 3, 8)):
        _raises(lambda: call(**ok, gate=gate), "gate has shape")
    for name in ("weight", "bias", "next_weight", "next_bias"):
        _raises(lambda: call(**ok, **{name: m(7)}), name + " has shape")
    _raises(lambda: call(**ok, after=False, weight=m(8)), "not the norm after the block")
    _raises(lambda: call(**ok, before=False, next_bias=m(8)), "not the norm before the next block")
    _raises(lambda: call(**ok, before=False, normed=m(6, 8)), "not the norm before the next block")
    _raises(lambda: call(**ok, after=False, before=False), "neither norm")
    _raises(lambda: call(**ok, eps=-1.0), "eps")
    for scale in (float("inf"), float("nan"), 1e300):
        _raises(lambda: call(**ok, scale=scale), "not a finite float32")
    _raises(lambda: call(**ok, out=m(5, 8)), "out has shape")
    _raises(lambda: call(**ok, normed=m(6, 9)), "normed has shape")
    _raises(lambda: call(**ok, stats=m(2, 6)), "stats has shape")


def test_block_norm_backward_checks(no_library):  # noqa: F811
    call = P.block_norm_backward
    ok = dict(dout=m(6, 8), dnormed=m(6, 8), x=m(6, 8), out=m(6, 8), stats=m(4, 6))
    _raises(lambda: call(**ok), "must be a GPU tensor")
    _raises(lambda: call(None, None, m(6, 8), m(6, 8), m(4, 6)), "neither dout nor dnormed")
    _raises(lambda: call(**{**ok, "dout": m(6, 7)}), "dout has shape")
    _raises(lambda: call(**{**ok, "x": None}), "x has shape")
    _raises(lambda: call(**{**ok, "out": None}), "out has shape")
    _raises(lambda: call(**{**ok, "stats": m(2, 6)}), "stats has shape")
    _raises(lambda: call(**ok, gate=m(5, 8)), "gate has shape")
    _raises(lambda: call(**ok, after=False, weight=m(8)), "not the norm after the block")
    _raises(lambda: call(**ok, after=False, dbias=m(8)), "not the norm after the block")
    _raises(lambda: call(**{**ok, "dnormed": None}, dnext_weight=m(8)), "not the norm before the next block")
    _raises(lambda: call(**{**ok, "dnormed": None, "out": None}, after=False), "neither norm")
    _raises(lambda: call(**ok, dx=m(6, 9)), "dx has shape")


@pytest.fixture
def library(ff_library, monkeypatch):  # noqa: F811
    monkeypatch.setattr(R, "_check_dev", lambda *a, **kw: None)
    return ff_library


def _tensors():
    """Every operator's tensors by name, and the names of its call's arguments in order."""
    z = torch.zeros
    i8 = lambda *s: z(*s, dtype=I8)  # noqa: E731
    r = z(2, dtype=torch.int64)
    return {
        "quantize": (dict(x=z(6, 300)), "dtype rows d x ldx group q ldq scale stream", {}),
        "dequantize": (dict(q=i8(6, 300), scale=z(6, 3)), "dtype rows d q ldq scale group out ldout stream", {}),
        "dense_int8": (dict(x=i8(6, 8), x_scale=z(6, 1), weight=i8(5, 8).t(), weight_scale=z(5, 1), bias=z(5), residual=z(6, 5),
                            out=z(6, 5)),
                       "dtype M K N x ldx x_scale weight ldw weight_scale bias act residual ldr out ldy ws ws_bytes stream", {}),
        "dense_backward_int8": (dict(dy=z(6, 5), x=i8(6, 300), x_scale=z(6, 3), weight=z(300, 5), pre=i8(6, 5), pre_scale=z(6, 1),
                                     dx=z(6, 300), dweight=z(300, 5), dbias=z(5)),
                                "dtype M K N dy lddy x ldx x_scale x_group weight ldw order pre ldp pre_scale pre_group act drop dx "
                                "lddx dweight lddw dbias ws ws_bytes stream", dict(act=2, dropout=(0.5, r))),
        "block_norm": (dict(x=z(6, 8), residual=z(6, 8), gate=z(3, 8), weight=z(8), bias=z(8), next_weight=z(8), next_bias=z(8),
                            out=z(6, 8), normed=z(6, 8), stats=z(4, 6)),
                       "dtype rows d desc x ldx residual ldr gate weight bias next_weight next_bias out ldo normed ldn stats stream",
                       {}),
        "block_norm_backward": (dict(dout=z(6, 8), dnormed=z(6, 8), x=z(6, 8), out=z(6, 8), stats=z(4, 6), gate=z(3, 8), weight=z(8),
                                     bias=z(8), next_weight=z(8), next_bias=z(8), dx=z(6, 8), dresidual=z(6, 8), dgate=z(3, 8),
                                     dweight=z(8), dbias=z(8), dnext_weight=z(8), dnext_bias=z(8)),
                                "dtype rows d desc dout lddo dnormed lddn x ldx out ldo stats gate weight bias next_weight dx lddx "
                                "dresidual lddr dgate dweight dbias dnext_weight dnext_bias ws ws_bytes stream", {})}


@pytest.mark.parametrize("op", _tensors())
def test_every_tensor_goes_to_its_place(library, op):
    tensors, names, more = _tensors()[op]
    getattr(P, op)(**tensors, **more)
    (name, args), names = library.calls[-1], names.split()
    assert name == "cliffconv_" + op and len(args) == len(names)
    args = dict(zip(names, args))
    for k, t in tensors.items():
        if k in args:
            assert args[k] == t.data_ptr(), k
        else:
            assert (op, k) == ("block_norm_backward", "next_bias")  # its gradient is wanted, not its values
    want = dict(rows=6, d=300, M=6, K=8 if op == "dense_int8" else 300, N=5, group=0 if op == "quantize" else 128, x_group=128,
                pre_group=0, order=0, ldx=300 if "int8" not in op or op[-4:] == "int8" and op != "dense_int8" else 8)
    if op.startswith("block_norm"):
        want.update(d=8, ldx=8)
    for k, v in want.items():
        assert args.get(k, v) == v, (k, args[k])
    declared = {}

    class Entry:
        def __init__(self, name):
            self.name = name

        def __setattr__(self, k, v):
            object.__setattr__(self, k, v)
            if k == "argtypes":
                declared[self.name] = len(v)
    lib = type("L", (), {n: Entry(n) for n in R.EXPORTED})()  # noqa: F811
    R.declare(lib)
    assert declared["cliffconv_" + op] == len(names)


@pytest.mark.parametrize("op", _tensors())
def test_buffers_are_the_streams_own(library, streams, op):  # noqa: F811
    # what a call on another stream writes is allocated for that one; what it reads may be
    # freed after the call, and is noted as used there
    outputs = ("q", "scale") if op == "quantize" else ("out", "normed", "stats", "dx", "dresidual", "dgate", "dweight", "dbias",
                                                       "dnext_weight", "dnext_bias")
    if op == "block_norm_backward":
        outputs = outputs[3:]
    for stream, name in ((None, "first"), (_Stream(), "handle 1234")):
        tensors, _, more = _tensors()[op]
        inputs = {k: t for k, t in tensors.items() if k not in outputs}
        streams["made"].clear()
        streams["recorded"].clear()
        plan = getattr(P, op + "_plan")(**inputs, **more, stream=stream)
        assert streams["made"] and {s for _, s in streams["made"]} == {name} and streams["current"] == "first"
        used = {p for p, _ in streams["made"]} | {t.data_ptr() for t in inputs.values()}
        used |= {more["dropout"][1].data_ptr()} if "dropout" in more else set()
        assert set(streams["recorded"]) == (set() if stream is None else {(p, "first") for p, _ in streams["made"]} |
                                            {(p, name) for p in used})
        streams["recorded"].clear()
        plan(7)
        assert set(streams["recorded"]) == {(p, "handle 7") for p in used}


@pytest.mark.parametrize("op", _tensors())
def test_tensors_that_require_a_gradient(library, monkeypatch, op):
    # autograd would not see the call: refused while it records, for each tensor
    for module in (F, R):
        monkeypatch.setattr(module, "_check_dev", lambda t, name, *a, **kw: F._check_grad(t, name))
    for name, t in _tensors()[op][0].items():
        tensors, _, more = _tensors()[op]
        if t.dtype != torch.float32:
            continue
        tensors[name].requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            getattr(P, op)(**tensors, **more)
        with torch.no_grad():
            getattr(P, op)(**tensors, **more)
    getattr(P, op)(**_tensors()[op][0], **more)


def test_orders_of_the_weight(library):
    z = torch.zeros
    with pytest.raises(ValueError, match="not the transposed view"):
        P.dense_int8(z(6, 8, dtype=I8), z(6, 1), z(8, 5, dtype=I8), z(5, 1))


# ---- the C ABI

E, S, A, O, W = P.CLIFF_EINVAL, P.CLIFF_ESHAPE, P.CLIFF_EALIGN, P.CLIFF_EOVERLAP, P.CLIFF_ESCRATCH

QUANT = dict(dtype=1, rows=4, d=300, x=FAKE, ldx=300, group=128, q=FAKE + MB, ldq=300, scale=FAKE + 2 * MB, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), E), (dict(x=None), E), (dict(q=None), E), (dict(scale=None), E), (dict(group=64), E), (dict(group=-1), E),
    (dict(rows=-1), S), (dict(d=0), S), (dict(ldx=299), S), (dict(ldq=299), S), (dict(rows=1 << 31), S), (dict(ldq=1 << 40), S),
    (dict(x=FAKE + 1), A), (dict(scale=FAKE + 2 * MB + 2), A),
    (dict(q=FAKE + 8), O), (dict(scale=FAKE), O), (dict(scale=FAKE + MB), O), (dict(q=FAKE + 2 * MB + 40), O),
], ids=str)
def test_quantize_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_quantize", QUANT, kw) == expect


BACK = dict(dtype=1, rows=4, d=300, q=FAKE, ldq=300, scale=FAKE + MB, group=128, y=FAKE + 2 * MB, ldy=300, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=-1), E), (dict(q=None), E), (dict(y=None), E), (dict(scale=None), E), (dict(group=1), E), (dict(d=0), S),
    (dict(ldy=299), S), (dict(y=FAKE + 2 * MB + 1), A), (dict(scale=FAKE + MB + 1), A), (dict(y=FAKE), O), (dict(y=FAKE + MB + 40), O),
], ids=str)
def test_dequantize_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_dequantize", BACK, kw) == expect


INT8 = dict(dtype=1, M=4, K=8, N=16, x=FAKE, ldx=8, xs=FAKE + MB, w=FAKE + 2 * MB, ldw=8, ws=FAKE + 3 * MB, bias=FAKE + 4 * MB, act=2,
            residual=FAKE + 5 * MB, ldr=16, y=FAKE + 6 * MB, ldy=16, space=FAKE + 7 * MB, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), E), (dict(x=None), E), (dict(xs=None), E), (dict(w=None), E), (dict(ws=None), E), (dict(y=None), E),
    (dict(act=4), E), (dict(act=-1), E), (dict(M=-1), S), (dict(K=0), S), (dict(N=0), S), (dict(K=131072, ldx=131072, ldw=131072), S),
    (dict(ldx=7), S), (dict(ldw=7), S), (dict(ldr=15), S), (dict(ldy=15), S), (dict(xs=FAKE + MB + 2), A), (dict(ws=FAKE + 3 * MB + 1), A),
    (dict(bias=FAKE + 4 * MB + 1), A), (dict(y=FAKE + 6 * MB + 1), A), (dict(y=FAKE), O), (dict(y=FAKE + 2 * MB), O),
    (dict(y=FAKE + MB), O), (dict(y=FAKE + 3 * MB), O), (dict(y=FAKE + 4 * MB), O), (dict(y=FAKE + 5 * MB + 2), O),
    (dict(M=70, K=4096, ldx=4096, ldw=4096, space=None), W), (dict(M=70, K=4096, ldx=4096, ldw=4096, bytes=16), W),
    (dict(M=70, K=4096, ldx=4096, ldw=4096, space=FAKE + 7 * MB + 4), A),
    (dict(M=70, K=4096, ldx=4096, ldw=4096, space=FAKE + 6 * MB), O),
], ids=str)
def test_dense_int8_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_dense_int8", INT8, kw) == expect


GRAD8 = dict(dtype=1, M=4, K=300, N=16, dy=FAKE, lddy=16, x=FAKE + MB, ldx=300, xs=FAKE + 2 * MB, xg=128, w=FAKE + 3 * MB, ldw=16,
             order=0, pre=FAKE + 4 * MB, ldp=16, ps=FAKE + 5 * MB, pg=0, act=2, drop=None, dx=FAKE + 6 * MB, lddx=300, dw=FAKE + 7 * MB,
             lddw=16, db=FAKE + 8 * MB, ws=FAKE + 9 * MB, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), E), (dict(dy=None), E), (dict(x=None), E), (dict(xs=None), E), (dict(w=None), E), (dict(pre=None), E),
    (dict(ps=None), E), (dict(xg=32), E), (dict(pg=1), E), (dict(act=9), E), (dict(order=2), E), (dict(drop=_drop(-0.1)), E),
    (dict(N=0), S), (dict(ldx=299), S), (dict(ldp=15), S), (dict(lddx=299), S), (dict(lddw=15), S), (dict(xs=FAKE + 2 * MB + 2), A),
    (dict(ps=FAKE + 5 * MB + 2), A), (dict(dw=FAKE + 7 * MB + 1), A), (dict(dx=FAKE + MB), O), (dict(dx=FAKE + 2 * MB), O),
    (dict(dw=FAKE + 4 * MB), O), (dict(dw=FAKE + 5 * MB), O), (dict(db=FAKE + 7 * MB + 2), O), (dict(ws=None), W), (dict(bytes=1), W),
    (dict(ws=FAKE + 9 * MB + 8), A), (dict(ws=FAKE + 6 * MB), O), (dict(ws=FAKE + 5 * MB), O),
], ids=str)
def test_dense_backward_int8_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_dense_backward_int8", GRAD8, kw) == expect


def _desc(after=1, before=1, rms=0, scale=1.0, eps=1e-5, gates=2):
    return ctypes.byref(R.CliffBlockNormDesc(after, before, rms, scale, eps, gates))


NORM = dict(dtype=1, rows=4, d=8, desc=_desc(), x=FAKE, ldx=8, res=FAKE + MB, ldr=8, gate=FAKE + 2 * MB, w=FAKE + 3 * MB, b=FAKE + 4 * MB,
            nw=FAKE + 5 * MB, nb=FAKE + 6 * MB, out=FAKE + 7 * MB, ldo=8, normed=FAKE + 8 * MB, ldn=8, stats=FAKE + 9 * MB, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), E), (dict(desc=None), E), (dict(x=None), E), (dict(res=None), E), (dict(out=None), E), (dict(normed=None), E),
    (dict(desc=_desc(after=0, before=0)), E), (dict(desc=_desc(after=0)), E), (dict(desc=_desc(before=0)), E),
    (dict(desc=_desc(eps=-1.0)), E), (dict(desc=_desc(eps=float("nan"))), E), (dict(desc=_desc(scale=float("inf"))), E),
    (dict(desc=_desc(scale=1e39)), E), (dict(desc=_desc(gates=3)), S), (dict(desc=_desc(gates=0)), S), (dict(desc=_desc(gates=-4)), S),
    (dict(rows=-1), S), (dict(d=0), S), (dict(ldx=7), S), (dict(ldr=7), S), (dict(ldo=7), S), (dict(ldn=7), S),
    (dict(x=FAKE + 1), A), (dict(gate=FAKE + 2 * MB + 1), A), (dict(stats=FAKE + 9 * MB + 2), A),
    (dict(out=FAKE + 8 * MB), O), (dict(out=FAKE + 2), O), (dict(out=FAKE, ldo=9), O), (dict(normed=FAKE + 2 * MB), O),
    (dict(stats=FAKE), O), (dict(stats=FAKE + MB), O), (dict(out=FAKE + 3 * MB), O), (dict(normed=FAKE + 9 * MB + 8), O),
], ids=str)
def test_block_norm_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_block_norm", NORM, kw) == expect


NGRAD = dict(dtype=1, rows=4, d=8, desc=_desc(), dout=FAKE, lddo=8, dn=FAKE + MB, lddn=8, x=FAKE + 2 * MB, ldx=8, out=FAKE + 3 * MB,
             ldo=8, stats=FAKE + 4 * MB, gate=FAKE + 5 * MB, w=FAKE + 6 * MB, b=FAKE + 7 * MB, nw=FAKE + 8 * MB, dx=FAKE + 9 * MB, lddx=8,
             dr=FAKE + 10 * MB, lddr=8, dg=FAKE + 11 * MB, dw=FAKE + 12 * MB, db=FAKE + 13 * MB, dnw=FAKE + 14 * MB, dnb=FAKE + 15 * MB,
             ws=FAKE + 16 * MB, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), E), (dict(desc=None), E), (dict(dn=None), E), (dict(x=None), E), (dict(out=None), E), (dict(stats=None), E),
    (dict(dx=None), E), (dict(dr=None), E), (dict(gate=None), E), (dict(desc=_desc(after=0)), E), (dict(desc=_desc(before=0)), E),
    (dict(desc=_desc(gates=3)), S), (dict(lddo=7), S), (dict(lddn=7), S), (dict(ldo=7), S), (dict(lddx=7), S), (dict(lddr=7), S),
    (dict(dg=FAKE + 11 * MB + 1), A), (dict(stats=FAKE + 4 * MB + 2), A), (dict(dx=FAKE + 10 * MB), O), (dict(dx=FAKE + 2 * MB), O),
    (dict(dr=FAKE + 3 * MB), O), (dict(dx=FAKE + 2), O), (dict(dr=FAKE + MB, lddr=9), O), (dict(dg=FAKE), O), (dict(dw=FAKE + 11 * MB), O),
    (dict(dnb=FAKE + 14 * MB + 2), O), (dict(dnw=FAKE + 4 * MB), O), (dict(ws=None), W), (dict(bytes=8), W),
    (dict(ws=FAKE + 16 * MB + 4), A), (dict(ws=FAKE + 9 * MB), O),
], ids=str)
def test_block_norm_backward_errors(lib, kw, expect):  # noqa: F811
    assert _call(lib, "cliffconv_block_norm_backward", NGRAD, kw) == expect


def test_no_rows_is_no_work(lib):  # noqa: F811
    assert _call(lib, "cliffconv_quantize", QUANT, dict(rows=0, x=None, q=None, scale=None)) == P.CLIFF_OK
    assert _call(lib, "cliffconv_dequantize", BACK, dict(rows=0, y=None, q=None, scale=None)) == P.CLIFF_OK
    assert _call(lib, "cliffconv_dense_int8", INT8, dict(M=0, x=None, xs=None, y=None, residual=None)) == P.CLIFF_OK
    assert _call(lib, "cliffconv_block_norm", NORM, dict(rows=0, x=None, res=None, out=None, normed=None, stats=None)) == P.CLIFF_OK


def test_workspace_sizes_of_bad_arguments(lib):  # noqa: F811
    assert lib.cliffconv_dense_int8_workspace(-1, 4, 4) == 0
    assert lib.cliffconv_dense_int8_workspace(70, 131072, 4) == 0
    assert lib.cliffconv_dense_backward_int8_workspace(9, 4, 4, 4) == 0
    assert lib.cliffconv_block_norm_backward_workspace(0, 4, 0, 1) == 0
    assert lib.cliffconv_block_norm_backward_workspace(0, 4, 8, -1) == 0
