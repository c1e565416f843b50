"""Refusals of the feed-forward operators, on the CPU: the binding's checks of
shape-only ("meta") tensors and the C ABI's checks of addresses that are never
dereferenced (each case carries a defect that the library must report before
any device work); and the tests' own generator against published words."""
import ctypes
import os

import pytest
import torch

import ff_oracle as O
import paper_2507_01040_amd as P
from paper_2507_01040_amd import feed_forward as F


def m(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


def _raises(fn, match):
    with pytest.raises(ValueError, match=match):
        fn()


@pytest.fixture
def no_library(monkeypatch):
    def fail(*a, **kw):
        raise AssertionError("the library was called")
    monkeypatch.setattr(P, "load", fail)


def test_generator_known_answers():
    # Philox4x32-7 of the all-zero and all-one inputs, as its authors publish them
    assert O.philox_words(0, 0, 1, 4)[0].tolist() == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    # counters: the column's quad, the row and the step
    a = O.philox_words(5, 9, 3, 11)
    assert a.shape == (3, 11)
    assert (O.philox_words(5, 9, 1, 11, first_row=2)[0] == a[2]).all()
    assert (O.philox_words(5, 10, 3, 11) != a).any()


def test_dense_checks(no_library):
    ok = dict(x=m(6, 8), weight=m(8, 5), bias=m(5))
    _raises(lambda: P.dense(**ok), "x must be a GPU tensor")
    _raises(lambda: P.dense(**{**ok, "weight": m(5, 8)}), "weight has shape")
    _raises(lambda: P.dense(**{**ok, "weight": m(8, 5, 1)}), "weight has shape")
    _raises(lambda: P.dense(**{**ok, "bias": m(8)}), "bias has shape")
    _raises(lambda: P.dense(**ok, act=4), "unknown activation")
    _raises(lambda: P.dense(**ok, residual=m(6, 8)), "residual has shape")
    _raises(lambda: P.dense(**ok, pre=m(5, 5)), "pre has shape")
    _raises(lambda: P.dense(**ok, out=m(5, 6)), "out has shape")
    _raises(lambda: P.dense(**ok, dropout=(1.5, m(2))), "probability")
    _raises(lambda: P.dense(**ok, dropout=(float("nan"), m(2))), "probability")
    _raises(lambda: P.dense(**ok, dropout=(0.5, m(3))), "rng has shape")
    _raises(lambda: P.dense(**{**ok, "x": m(6, 0)}), "x has shape")


def test_dense_backward_checks(no_library):
    ok = dict(dy=m(6, 5), x=m(6, 8), weight=m(8, 5))
    _raises(lambda: P.dense_backward(**ok), "dy must be a GPU tensor")
    _raises(lambda: P.dense_backward(**{**ok, "dy": m(6, 8)}), "dy has shape")
    _raises(lambda: P.dense_backward(**{**ok, "weight": m(5, 8)}), "weight has shape")
    _raises(lambda: P.dense_backward(**ok, act=P.ACT_GELU), "needs the pre-activations")
    _raises(lambda: P.dense_backward(**ok, act=P.ACT_GELU, pre=m(6, 8)), "pre has shape")
    _raises(lambda: P.dense_backward(**ok, dx=m(6, 5)), "dx has shape")
    _raises(lambda: P.dense_backward(**ok, dweight=m(5, 8)), "dweight has shape")
    _raises(lambda: P.dense_backward(**ok, dbias=m(8)), "dbias has shape")


def test_norm_and_dropout_checks(no_library):
    _raises(lambda: P.layer_norm(m(4, 8)), "x must be a GPU tensor")
    _raises(lambda: P.layer_norm(m(4, 8), m(4)), "weight has shape")
    _raises(lambda: P.layer_norm(m(4, 8), None, m(9)), "bias has shape")
    _raises(lambda: P.layer_norm(m(4, 8), eps=-1.0), "eps")
    _raises(lambda: P.layer_norm(m(4, 8), out=m(8, 4)), "out has shape")
    _raises(lambda: P.layer_norm(m(4, 8), mean=m(8)), "mean has shape")
    ok = dict(dy=m(4, 8), x=m(4, 8), mean=m(4), rstd=m(4))
    _raises(lambda: P.layer_norm_backward(**ok), "dy must be a GPU tensor")
    _raises(lambda: P.layer_norm_backward(**{**ok, "dy": m(4, 9)}), "dy has shape")
    _raises(lambda: P.layer_norm_backward(**{**ok, "rstd": m(8)}), "rstd has shape")
    _raises(lambda: P.layer_norm_backward(**ok, dresidual=m(8, 4)), "dresidual has shape")
    _raises(lambda: P.layer_norm_backward(**ok, dweight=m(4)), "dweight has shape")
    _raises(lambda: P.dropout(m(4, 8), 0.5, m(2)), "x must be a GPU tensor")
    _raises(lambda: P.dropout(m(4, 8), -0.5, m(2)), "probability")
    _raises(lambda: P.dropout(m(4, 8), 0.5, m(1)), "rng has shape")
    _raises(lambda: P.dropout(m(4, 8), 0.5, m(2), residual=m(8)), "residual has shape")


def test_row_strides():
    s = lambda t: F._row_stride(t, "t")  # noqa: E731
    assert s(torch.empty(4, 8)) == 8
    assert s(torch.empty(4, 12)[:, 2:10]) == 12
    assert s(torch.empty(3, 4, 12)[..., :8]) == 12
    assert s(torch.empty(3, 1, 8)) == 8
    assert s(torch.empty(8)) == 8
    assert s(torch.empty(1, 8)[:, :3]) == 3   # one row: any stride will do
    assert s(torch.empty(6, 4, 8)[:, 1]) == 32
    assert s(torch.empty(5, 1)) == 1
    assert s(torch.empty(0, 8)) == 8
    _raises(lambda: s(torch.empty(8, 4).t()), "features are not contiguous")
    _raises(lambda: s(torch.empty(1, 8).expand(4, 8)), "rows overlap")
    _raises(lambda: s(torch.empty(3, 4, 8)[:, :2]), "no single stride")
    o = F._weight_order
    assert o(torch.empty(8, 5)) == (0, 5)
    assert o(torch.empty(5, 8).t()) == (1, 8)
    assert o(torch.empty(8, 9)[:, :5]) == (0, 9)
    assert o(torch.empty(1, 5)) == (0, 5)
    assert o(torch.empty(8, 1)) == (0, 1)
    _raises(lambda: o(torch.empty(8, 10)[:, ::2]), "neither axis")
    _raises(lambda: o(torch.empty(1, 5).expand(8, 5)), "neither axis")


FAKE = 0x7F0000000000  # never dereferenced
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("addresses that do not exist: for machines without a GPU")
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("libcliffconv.so not built")
    return P.load()


def _call(lib, fn, base, kw):
    args = dict(base)
    for k, v in kw.items():
        assert k in args, k
        args[k] = v
    return getattr(lib, fn)(*args.values())


def _drop(p=0.5, rng=FAKE + 20 * MB):
    d = F.CliffDropoutDesc()
    d.p, d.rng = p, rng
    return ctypes.byref(d)


DENSE = dict(dtype=1, M=4, K=8, N=16, x=FAKE, ldx=8, w=FAKE + MB, ldw=16, order=0, bias=FAKE + 2 * MB,
             act=2, drop=None, residual=FAKE + 3 * MB, ldr=16, pre=FAKE + 4 * MB, ldp=16,
             y=FAKE + 5 * MB, ldy=16, ws=FAKE + 6 * MB, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), P.CLIFF_EINVAL), (dict(dtype=-1), P.CLIFF_EINVAL),
    (dict(x=None), P.CLIFF_EINVAL), (dict(w=None), P.CLIFF_EINVAL), (dict(y=None), P.CLIFF_EINVAL),
    (dict(act=4), P.CLIFF_EINVAL), (dict(order=2), P.CLIFF_EINVAL),
    (dict(drop=_drop(1.5)), P.CLIFF_EINVAL), (dict(drop=_drop(float("nan"))), P.CLIFF_EINVAL),
    (dict(drop=_drop(0.5, None)), P.CLIFF_EINVAL),
    (dict(M=-1), P.CLIFF_ESHAPE), (dict(K=0), P.CLIFF_ESHAPE), (dict(N=0), P.CLIFF_ESHAPE),
    (dict(M=1 << 31), P.CLIFF_ESHAPE), (dict(M=1 << 30, K=1 << 20, ldx=1 << 20), P.CLIFF_ESHAPE),
    (dict(ldx=7), P.CLIFF_ESHAPE), (dict(ldw=15), P.CLIFF_ESHAPE), (dict(ldy=15), P.CLIFF_ESHAPE),
    (dict(ldr=15), P.CLIFF_ESHAPE), (dict(ldp=1), P.CLIFF_ESHAPE), (dict(ldx=1 << 40), P.CLIFF_ESHAPE),
    (dict(order=1, ldw=7), P.CLIFF_ESHAPE),
    (dict(x=FAKE + 1), P.CLIFF_EALIGN), (dict(dtype=0, y=FAKE + 5 * MB + 2), P.CLIFF_EALIGN),
    (dict(drop=_drop(0.5, FAKE + 20 * MB + 4)), P.CLIFF_EALIGN),
    (dict(y=FAKE), P.CLIFF_EOVERLAP), (dict(y=FAKE + 3 * MB + 2), P.CLIFF_EOVERLAP),
    (dict(y=FAKE + 3 * MB, ldy=17), P.CLIFF_EOVERLAP), (dict(pre=FAKE + 5 * MB), P.CLIFF_EOVERLAP),
    (dict(pre=FAKE + 3 * MB), P.CLIFF_EOVERLAP), (dict(drop=_drop(0.5, FAKE + 5 * MB + 8)), P.CLIFF_EOVERLAP),
    # two column ranges of one buffer that share a column
    (dict(x=FAKE, ldx=32, y=FAKE + 14, ldy=32, residual=None), P.CLIFF_EOVERLAP),
], ids=str)
def test_dense_errors(lib, kw, expect):
    assert _call(lib, "cliffconv_dense", DENSE, kw) == expect


GRAD = dict(dtype=1, M=4, K=8, N=16, dy=FAKE, lddy=16, x=FAKE + MB, ldx=8, w=FAKE + 2 * MB, ldw=16, order=0,
            pre=FAKE + 3 * MB, ldp=16, act=2, drop=None, dx=FAKE + 4 * MB, lddx=8, dw=FAKE + 5 * MB, lddw=16,
            db=FAKE + 6 * MB, ws=FAKE + 7 * MB, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=3), P.CLIFF_EINVAL), (dict(dy=None), P.CLIFF_EINVAL), (dict(x=None), P.CLIFF_EINVAL),
    (dict(w=None), P.CLIFF_EINVAL), (dict(pre=None), P.CLIFF_EINVAL), (dict(act=-1), P.CLIFF_EINVAL),
    (dict(drop=_drop(-0.1)), P.CLIFF_EINVAL), (dict(N=0), P.CLIFF_ESHAPE), (dict(lddx=7), P.CLIFF_ESHAPE),
    (dict(lddw=15), P.CLIFF_ESHAPE), (dict(lddy=15), P.CLIFF_ESHAPE), (dict(dw=FAKE + 5 * MB + 1), P.CLIFF_EALIGN),
    (dict(dx=FAKE + MB), P.CLIFF_EOVERLAP), (dict(dw=FAKE + 2 * MB), P.CLIFF_EOVERLAP),
    (dict(db=FAKE + 5 * MB + 2), P.CLIFF_EOVERLAP), (dict(dx=FAKE), P.CLIFF_EOVERLAP),
    (dict(ws=None), P.CLIFF_ESCRATCH), (dict(ws_bytes=1), P.CLIFF_ESCRATCH),
    (dict(ws=FAKE + 7 * MB + 8), P.CLIFF_EALIGN), (dict(ws=FAKE + 4 * MB), P.CLIFF_EOVERLAP),
], ids=str)
def test_dense_backward_errors(lib, kw, expect):
    assert _call(lib, "cliffconv_dense_backward", GRAD, kw) == expect


NORM = dict(dtype=1, rows=4, d=8, x=FAKE, ldx=8, w=FAKE + MB, b=FAKE + 2 * MB, eps=1e-5, y=FAKE + 3 * MB, ldy=8,
            mean=FAKE + 4 * MB, rstd=FAKE + 5 * MB, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dtype=9), P.CLIFF_EINVAL), (dict(x=None), P.CLIFF_EINVAL), (dict(y=None), P.CLIFF_EINVAL),
    (dict(eps=-1e-9), P.CLIFF_EINVAL), (dict(eps=float("nan")), P.CLIFF_EINVAL), (dict(rows=-1), P.CLIFF_ESHAPE),
    (dict(d=0), P.CLIFF_ESHAPE), (dict(ldx=7), P.CLIFF_ESHAPE), (dict(mean=FAKE + 4 * MB + 2), P.CLIFF_EALIGN),
    (dict(y=FAKE + 2), P.CLIFF_EOVERLAP), (dict(y=FAKE, ldy=9), P.CLIFF_EOVERLAP), (dict(y=FAKE + MB), P.CLIFF_EOVERLAP),
    (dict(rstd=FAKE + 4 * MB + 12), P.CLIFF_EOVERLAP), (dict(mean=FAKE), P.CLIFF_EOVERLAP),
], ids=str)
def test_layer_norm_errors(lib, kw, expect):
    assert _call(lib, "cliffconv_layer_norm", NORM, kw) == expect


NGRAD = dict(dtype=1, rows=4, d=8, dy=FAKE, lddy=8, x=FAKE + MB, ldx=8, mean=FAKE + 2 * MB, rstd=FAKE + 3 * MB,
             w=FAKE + 4 * MB, res=FAKE + 5 * MB, ldr=8, dx=FAKE + 6 * MB, lddx=8, dw=FAKE + 7 * MB, db=FAKE + 8 * MB,
             ws=FAKE + 9 * MB, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(dy=None), P.CLIFF_EINVAL), (dict(mean=None), P.CLIFF_EINVAL), (dict(dx=None), P.CLIFF_EINVAL),
    (dict(d=0), P.CLIFF_ESHAPE), (dict(ldr=7), P.CLIFF_ESHAPE), (dict(dx=FAKE + 6 * MB + 1), P.CLIFF_EALIGN),
    (dict(dx=FAKE + MB), P.CLIFF_EOVERLAP), (dict(dx=FAKE + 2), P.CLIFF_EOVERLAP), (dict(dw=FAKE), P.CLIFF_EOVERLAP),
    (dict(db=FAKE + 7 * MB), P.CLIFF_EOVERLAP), (dict(ws=None), P.CLIFF_ESCRATCH), (dict(ws_bytes=8), P.CLIFF_ESCRATCH),
    (dict(ws=FAKE + 6 * MB), P.CLIFF_EOVERLAP),
], ids=str)
def test_layer_norm_backward_errors(lib, kw, expect):
    assert _call(lib, "cliffconv_layer_norm_backward", NGRAD, kw) == expect


DROP = dict(dtype=1, rows=4, d=8, x=FAKE, ldx=8, drop=_drop(), res=FAKE + MB, ldr=8, y=FAKE + 2 * MB, ldy=8, stream=None)


@pytest.mark.parametrize("kw,expect", [
    (dict(drop=None), P.CLIFF_EINVAL), (dict(x=None), P.CLIFF_EINVAL), (dict(drop=_drop(2.0)), P.CLIFF_EINVAL),
    (dict(d=0), P.CLIFF_ESHAPE), (dict(ldy=3), P.CLIFF_ESHAPE), (dict(y=FAKE + 1), P.CLIFF_EALIGN),
    (dict(y=FAKE + 2), P.CLIFF_EOVERLAP), (dict(y=FAKE + MB, ldy=16), P.CLIFF_EOVERLAP),
    (dict(y=FAKE + 20 * MB), P.CLIFF_EOVERLAP),
], ids=str)
def test_dropout_errors(lib, kw, expect):
    assert _call(lib, "cliffconv_dropout", DROP, kw) == expect


def test_no_rows_is_no_work(lib):
    none = dict(x=None, y=None, residual=None, pre=None)
    assert _call(lib, "cliffconv_dense", DENSE, dict(M=0, **none)) == P.CLIFF_OK
    assert _call(lib, "cliffconv_layer_norm", NORM, dict(rows=0, x=None, y=None)) == P.CLIFF_OK
    assert _call(lib, "cliffconv_dropout", DROP, dict(rows=0, x=None, y=None)) == P.CLIFF_OK


def test_workspace_sizes_of_bad_arguments(lib):
    assert lib.cliffconv_dense_workspace(7, 4, 4, 4) == 0
    assert lib.cliffconv_dense_workspace(0, -1, 4, 4) == 0
    assert lib.cliffconv_dense_backward_workspace(0, 1 << 30, 1, 1 << 30) == 0
    assert lib.cliffconv_layer_norm_backward_workspace(0, 4, 0) == 0
