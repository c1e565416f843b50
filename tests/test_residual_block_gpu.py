"""The 8-bit operators and the block norm on the GPU against plain implementations in
64 bits (block_oracle.py, which derives the bounds; integers and scales exactly)."""
import itertools

import pytest
import torch

import block_oracle as B
import ff_oracle as O
import paper_2507_01040_amd as P
from test_feed_forward_gpu import DTYPES, Draw, KEY, STEP, guarded, ids, rng

pytestmark = pytest.mark.gpu
EPS = 1e-5


def exactly(q, scale, x, group):
    want, ws = B.quantize(x.reshape(-1, x.shape[-1]), group)
    assert torch.equal(q.cpu().double().reshape(want.shape), want)
    assert torch.equal(scale.cpu().view(torch.int32)[~torch.isnan(ws)], ws.view(torch.int32)[~torch.isnan(ws)])
    assert torch.equal(torch.isnan(scale.cpu()), torch.isnan(ws))


ROWS = [(1, 1), (1, 4096), (3, 7), (5, 128), (7, 129), (300, 8), (33, 777), (64, 1024), (17, 2049), (4, 8192), (3, 8193), (2, 20001),
        (4099, 128), (1001, 260), (1100, 2100), (700, 5000)]


@pytest.mark.parametrize("group", [None, 128])
@pytest.mark.parametrize("size", ROWS, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize(dtype, size, group):
    x = Draw(1, dtype).rows(*size, pad=size[0] % 3)
    q, scale = P.quantize(x, group=group)
    exactly(q, scale, x, group)
    for out in DTYPES:
        O.check(P.dequantize(q, scale, dtype=out), B.dequantize(q, scale, out), "values")


@pytest.mark.parametrize("group", [None, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize_next_to_the_border_of_two_integers(dtype, group):
    # quotients in the middle of two integers, and the floats around them
    x = torch.zeros(64, 256, dtype=torch.float64)
    for r in range(64):
        s = 1.0 + r / 64 if r % 2 else 2.0 ** (r - 32)
        scale = (torch.tensor(127 * s).to(dtype).double() / 127).float().double()
        half = ((torch.arange(256) % 253 - 126).double() + 0.5) * scale
        v = half.to(dtype)
        v = v.view({4: torch.int32, 2: torch.int16}[v.element_size()])
        v = (v + (torch.arange(256) // 3 % 3 - 1).to(v.dtype)).view(dtype)
        x[r] = v.double()
        x[r, 0] = x[r, 128] = torch.tensor(127 * s).to(dtype).double()
    x = x.to(dtype).cuda()
    exactly(*P.quantize(x, group=group), x, group)


@pytest.mark.parametrize("group", [None, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize_extremes(dtype, group):
    big = torch.finfo(dtype).max
    x = Draw(2, dtype).rows(40, 300)
    x[0] = 0.0
    x[1, 5] = float("inf")
    x[2, 299] = float("nan")
    x[3, 130] = -float("inf")
    x[4] = big
    x[5] = -big
    x[6, :] = torch.finfo(dtype).tiny
    x[7, :] = torch.finfo(dtype).smallest_normal * 0.37
    x[8, ::2] = torch.finfo(dtype).tiny * 130
    x[9, 3] = big
    q, scale = P.quantize(x, group=group)
    exactly(q, scale, x, group)
    y = P.dequantize(q, scale, dtype=torch.float32)
    assert bool(torch.isnan(y[1, :128]).all() and torch.isnan(y[3]).any()) and bool((y[0] == 0).all())


def test_rows_between_others_stay():
    for dtype, group in itertools.product(DTYPES, (None, 128)):
        x = Draw(3, dtype).rows(13, 301, pad=2)
        q, q_intact = guarded(13, 301, torch.int8)
        scale = torch.empty(13, 3 if group else 1, device="cuda:0")
        assert P.quantize(x, group=group, q=q, scale=scale)[0] is q
        exactly(q, scale, x, group)
        y, intact = guarded(13, 301, dtype)
        assert P.dequantize(q, scale, out=y) is y and intact() and q_intact()
        O.check(y, B.dequantize(q, scale, dtype), "values")


class Eight(Draw):
    def int8(self, n, d, pad=0, offset=0):
        v = torch.from_numpy(self.rng.integers(-127, 128, (n, d + pad + offset)))
        return v.to(torch.int8).to("cuda:0")[:, offset:offset + d]

    def scale(self, n, groups=1, size=1.0):
        return torch.from_numpy(self.rng.uniform(0.5 * size, 1.5 * size, (n, groups))).float().to("cuda:0")


# (M, K, N): one row, few, around the tiles' edges, long sums, wide outputs
SIZES = [(1, 64, 64), (1, 1, 1), (3, 7, 5), (1, 4096, 512), (2, 520, 1000), (16, 2048, 96), (17, 96, 129), (24, 1024, 256), (32, 64, 72),
         (33, 65, 63), (64, 256, 128), (65, 16, 257), (127, 136, 320), (128, 128, 128), (130, 1040, 264), (255, 64, 511),
         (256, 512, 256), (257, 208, 513), (520, 784, 1032), (1000, 33, 40), (4099, 64, 24), (9, 3001, 16), (300, 16384, 8),
         (520, 2064, 1024), (20000, 128, 200), (16390, 100, 130), (64, 16384, 48), (2050, 17, 1030), (9001, 112, 257)]


def _int8(dtype, size, i, pad=0, offset=0):
    M, K, N = size
    v = Eight(4, dtype)
    x, w = v.int8(M, K, pad, offset), v.int8(N, K, pad, offset)
    xs, ws = v.scale(M), v.scale(N, size=1 / (5000 * K ** 0.5))
    b = v.vector(N) if i % 3 else None
    res = v.rows(M, N, pad=pad) if i % 2 else None
    y, intact = guarded(M, N, dtype, pad=(3, 0, 8)[i % 3])
    got = P.dense_int8(x, xs, w.t(), ws, b, act=i % 4, residual=res, out=y)
    assert got is y and intact()
    O.check(y, B.dense_int8(x, xs, w.t(), ws, b, i % 4, res, dtype), "y")


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_int8(dtype, size):
    _int8(dtype, size, SIZES.index(size))
    _int8(dtype, size, SIZES.index(size) + 1, pad=5)


@pytest.mark.parametrize("size", [(1, 256, 96), (24, 1024, 256), (130, 1040, 264), (520, 784, 1032), (16390, 112, 130)], ids=str)
@pytest.mark.parametrize("pad,offset", [(16, 0), (16, 16), (0, 1), (15, 1), (32, 3)])
def test_dense_int8_alignment(size, pad, offset):
    for i, dtype in enumerate(DTYPES):
        _int8(dtype, size, i, pad, offset)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_int8_largest_sums(dtype):
    # -128 times -128 over the longest contraction, and its sums of alternating signs
    K = 131071
    x = torch.full((40, K), -128, dtype=torch.int8, device="cuda:0")
    w = torch.full((3, K), -128, dtype=torch.int8, device="cuda:0")
    w[1, ::2] = 127
    w[2] = 127
    one, small = torch.ones(40, 1, device="cuda:0"), torch.full((3, 1), 2.0 ** -20, device="cuda:0")
    O.check(P.dense_int8(x, one, w.t(), small, dtype=dtype), B.dense_int8(x, one, w.t(), small, None, 0, None, dtype), "y")
    O.check(P.dense_int8(x[:3], one[:3], w.t(), small, dtype=dtype),
            B.dense_int8(x[:3], one[:3], w.t(), small, None, 0, None, dtype), "y of few rows")


@pytest.mark.parametrize("M", [3, 40, 300])
def test_dense_int8_scales_that_are_not_finite(M):
    # a NaN scale (a row or weight that held an infinity) makes NaN of its row or column
    # and of nothing else; scales whose product leaves fp32 do not
    v = Eight(5, torch.float32)
    x, w, xs, ws = v.int8(M, 200), v.int8(70, 200), v.scale(M), v.scale(70, size=1e-4)
    xs[1], ws[3] = float("nan"), float("nan")
    xs[0], ws[5], ws[6] = 2.0 ** 120, 2.0 ** -126, 2.0 ** -60
    x[0, :] = 0
    x[0, :9] = 100
    y = P.dense_int8(x, xs, w.t(), ws, dtype=torch.float32)
    want = B.dense_int8(x, xs, w.t(), ws, None, 0, None, torch.float32)
    inside = want[0].abs() < 3e38
    assert bool(inside[0, 5] and inside[0, 6])
    big = ~inside & ~torch.isnan(want[0])
    O.check(torch.where(big.cuda(), 0.0, y), (torch.where(big, 0.0, want[0]), torch.where(big, 0.0, want[1])), "y")


BACKWARD = [(1, 1, 1), (1, 64, 72), (3, 7, 5), (33, 129, 65), (130, 72, 136), (256, 512, 256), (257, 300, 1), (1000, 33, 40),
            (4099, 64, 24), (520, 776, 1032), (3000, 128, 260)]


@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", BACKWARD, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_backward_int8(dtype, size, order):
    M, K, N = size
    i = BACKWARD.index(size) + (order == "oi")
    v = Eight(6, dtype)
    xg, pg = (-(-K // 128) if i % 2 else 1), (-(-N // 128) if i % 3 else 1)
    x, xs = v.int8(M, K, pad=i % 4), v.scale(M, xg, 0.01)
    pre, ps = v.int8(M, N), v.scale(M, pg, 0.01)
    w, dy = v.weight(K, N, order), v.rows(M, N, pad=i % 2)
    drop = (0.3, rng()) if i % 2 else None
    a = i % 4
    dx, dw, db = P.dense_backward_int8(dy, x, xs, w, pre if a else None, ps if a else None, act=a, dropout=drop)
    assert dw.stride() == w.stride() or 1 in (K, N)
    want = B.dense_backward_int8(dy, x, xs, w, pre, ps, a, drop and (0.3, (KEY, STEP)), dtype)
    for got, ref, name in zip((dx, dw, db), want, ("dx", "dw", "dbias")):
        O.check(got, ref, name)
    only = P.dense_backward_int8(dy, x, xs, w, pre if a else None, ps if a else None, act=a, dropout=drop, dx=False, bias=False)
    assert len(only) == 1 and torch.equal(only[0], dw)


def _norm_case(dtype, size, i, **kw):
    R, d = size
    v = Draw(7, dtype)
    gates = (0, 1, 2, R)[i % 4]
    if gates and R % gates:
        gates = 1
    after, before = ((True, True), (True, False), (True, True), (False, True))[i % 4 if i % 5 else 0]
    c = dict(x=v.rows(R, d, pad=i % 3, scale=1.5, shift=0.7), residual=v.rows(R, d, pad=i % 2), gate=None,
             scale=(1.0, 0.5, -2.0)[i % 3], weight=v.vector(d, 0.3, 1.0), bias=v.vector(d), next_weight=v.vector(d, 0.3, 1.0),
             next_bias=v.vector(d), after=after, before=before, rms=i % 2 == 1)
    if gates:
        c["gate"] = v.vector(d) if gates == 1 else v.rows(gates, d)
    if not after or i % 7 == 3:
        c["weight"] = c["bias"] = None
    if not before or i % 7 == 4:
        c["next_weight"] = c["next_bias"] = None
    if i % 3 == 1:
        c["bias"] = c["next_bias"] = None
    c.update(kw)
    return c


def _check_norm(c, got, dtype):
    want = B.block_norm(c["x"], c["residual"], c["gate"], c["scale"], c["weight"], c["bias"], c["next_weight"], c["next_bias"],
                        c["after"], c["before"], c["rms"], EPS, dtype)
    O.check(got[0], want[0], "out")
    if c["before"]:
        O.check(got[1], want[1], "normed")
    stats = got[-1][0 if c["after"] else 2:4 if c["before"] else 2]
    for s, w in zip(stats, want[2]):
        O.check(s, w, "statistics")


@pytest.mark.parametrize("size", ROWS, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm(dtype, size):
    for i in range(5):
        c = _norm_case(dtype, size, i + ROWS.index(size))
        _check_norm(c, P.block_norm(**c, eps=EPS), dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_in_place(dtype):
    for i, size in enumerate(((5, 128), (33, 777), (4, 8192), (2, 20001), (1001, 260))):
        c = _norm_case(dtype, size, 4 * i, after=True, before=True)
        want = P.block_norm(**c)
        for to in (("residual", "x"), ("x", "residual"), ("residual", None), (None, "x")):
            k = dict(c, x=c["x"].clone(), residual=c["residual"].clone())
            got = P.block_norm(**k, out=k.get(to[0]), normed=k.get(to[1]))
            for g, w in zip(got, want):
                assert torch.equal(g, w)


def _gradient(c, size, dtype, i):
    R, d = size
    v = Draw(8, dtype)
    before = c["before"]
    k = {n: c[n] for n in ("x", "gate", "scale", "weight", "bias", "next_weight", "next_bias", "after", "rms")}
    k["dout"] = v.rows(R, d, pad=i % 2) if not before or i % 3 else None
    k["dnormed"] = v.rows(R, d, pad=i % 3) if before else None
    k["out"] = v.rows(R, d, scale=1.5, shift=0.3) if before else None
    stats = torch.zeros(4, R, device="cuda:0")
    for n, t in ((0, k["x"] if c["after"] else None), (2, k["out"])):
        if t is not None:
            t = t.double()
            m = torch.zeros(R, device="cuda:0", dtype=torch.float64) if c["rms"] else t.mean(1)
            stats[n] = m
            stats[n + 1] = (((t - m[:, None]) ** 2).mean(1) + EPS) ** -0.5
    k["stats"] = stats
    return k


def _check_gradient(k, got, dtype):
    want = B.block_norm_backward(k["dout"], k["dnormed"], k["x"], k["out"], k["stats"], k["gate"], k["scale"], k["weight"], k["bias"],
                                 k["next_weight"], k["after"], k["rms"], dtype)
    for name, of in zip(got._fields, (k["x"], k["x"], k["gate"], k["weight"], k["bias"], k["next_weight"], k["next_bias"])):
        g = getattr(got, name)
        assert (g is None) == (of is None), name
        if g is not None:
            O.check(g, want[name], name)


@pytest.mark.parametrize("size", ROWS, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_gradient(dtype, size):
    for i in range(5):
        j = i + ROWS.index(size)
        k = _gradient(_norm_case(dtype, size, j), size, dtype, j)
        _check_gradient(k, P.block_norm_backward(**k), dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_gradient_in_place(dtype):
    for i, size in enumerate(((5, 128), (33, 777), (4, 8192), (2, 20001), (1001, 260))):
        k = _gradient(_norm_case(dtype, size, 4 * i, after=True, before=True), size, dtype, 1)
        want = P.block_norm_backward(**k)
        for to in (("dout", "dnormed"), ("dnormed", "dout")):
            m = dict(k, dout=k["dout"].clone(), dnormed=k["dnormed"].clone())
            got = P.block_norm_backward(**m, dx=m[to[0]], dresidual=m[to[1]])
            assert got.dx is m[to[0]]
            for g, w in zip(got, want):
                assert (g is None and w is None) or torch.equal(g, w)
        alone = P.block_norm_backward(**k, params=False)
        assert torch.equal(alone.dx, want.dx) and torch.equal(alone.dresidual, want.dresidual) and alone[2:] == (None,) * 5


@pytest.mark.parametrize("size", [r for r in ROWS if r[0]], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_gradient_with_a_gate_for_every_row(dtype, size):
    for i, (after, before) in enumerate(((True, True), (True, False), (False, True))):
        c = _norm_case(dtype, size, 4 + i, after=after, before=before, gate=Draw(9, dtype).rows(*size))
        if not after:
            c["weight"] = c["bias"] = None
        if not before:
            c["next_weight"] = c["next_bias"] = None
        k = _gradient(c, size, dtype, i)
        got = P.block_norm_backward(**k)
        _check_gradient(k, got, dtype)
        again = P.block_norm_backward(**k)
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gates", [1, 3])
def test_block_norm_gradient_against_differences(gates, rms):
    # of the fp32 kernels alone: the slope of a weighted sum of both outputs along one
    # direction of every input.  The outputs' errors are below 1e-5 of them (bounds of
    # block_oracle.py at these sizes), the step's third-order term below 1e-4 of the slope
    v = Draw(9, torch.float32)
    R, d, h = 6, 96, 2.0 ** -6
    inputs = dict(x=v.rows(R, d), residual=v.rows(R, d), gate=v.rows(gates, d) if gates > 1 else v.vector(d), weight=v.vector(d, 0.3, 1.0),
                  bias=v.vector(d), next_weight=v.vector(d, 0.3, 1.0), next_bias=v.vector(d))
    dout, dnormed = v.rows(R, d), v.rows(R, d)

    def loss(k):
        out, normed, _ = P.block_norm(**k, scale=0.7, rms=rms)
        return (out.double() * dout.double()).sum() + (normed.double() * dnormed.double()).sum()
    out, _, stats = P.block_norm(**inputs, scale=0.7, rms=rms)
    rest = {n: inputs[n] for n in ("x", "gate", "weight", "bias", "next_weight", "next_bias")}
    grads = P.block_norm_backward(dout, dnormed, out=out, stats=stats, scale=0.7, rms=rms, **rest)
    for name, g in zip(("x", "residual", "gate", "weight", "bias", "next_weight", "next_bias"), grads):
        along = v.rows(*inputs[name].reshape(-1, d).shape).reshape(inputs[name].shape)
        step = [loss(dict(inputs, **{name: inputs[name] + s * along})) for s in (h, -h, 2 * h, -2 * h)]
        slope = (8 * (step[0] - step[1]) - (step[2] - step[3])) / (12 * h)  # fourth order
        want = (g.double() * along.double()).sum()
        size = float((g.double() * along.double()).abs().sum())
        assert abs(float(slope - want)) < 2e-3 * size, name
