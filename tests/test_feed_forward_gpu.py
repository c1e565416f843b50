"""Dense layers, layer norm, dropout and their gradients on the GPU against
plain implementations in 64 bits (ff_oracle.py, which derives the bounds)."""
import itertools

import numpy as np
import pytest
import torch

import ff_oracle as O
import paper_2507_01040_amd as P

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}
ids = lambda v: IDS.get(v, str(v))  # noqa: E731
KEY, STEP = 0x123456789ABCDEF, 77


class Draw:
    def __init__(self, seed, dtype):
        self.rng, self.dtype = np.random.default_rng(seed), dtype

    def rows(self, n, d, pad=0, scale=1.0, shift=0.0, offset=0):
        v = self.rng.standard_normal((n, d + pad + offset)) * scale + shift
        return torch.from_numpy(v).to(self.dtype).to("cuda:0")[:, offset:offset + d]

    def vector(self, d, scale=1.0, shift=0.0):
        return self.rows(1, d, 0, scale, shift).reshape(d).contiguous()

    def weight(self, K, N, order):
        return self.rows(K, N, 0, K ** -0.5) if order == "io" else self.rows(N, K, 0, K ** -0.5).t()


def rng(key=KEY, step=STEP):
    return torch.tensor([key, step], dtype=torch.int64, device="cuda:0")


def guarded(n, d, dtype, pad=3):
    """A view [n, d] inside a larger buffer, and a check that nothing around it changed."""
    buf = torch.full((n + 2, d + pad), 7.0, dtype=dtype, device="cuda:0")
    view = buf[1:n + 1, :d]

    def intact():
        c = buf.clone()
        c[1:n + 1, :d] = 7.0
        return bool((c == 7.0).all())
    return view, intact


# (M, K, N): one row, few, around the tiles' edges, long sums, wide outputs
SIZES = [(1, 64, 64), (1, 1, 1), (3, 7, 5), (1, 1024, 512), (2, 520, 1000), (17, 96, 129), (24, 512, 256),
         (32, 64, 72), (33, 65, 63), (64, 256, 128), (65, 8, 257), (127, 136, 320), (128, 128, 128),
         (130, 1032, 264), (255, 64, 511), (256, 512, 256), (257, 200, 513), (520, 776, 1032),
         (1000, 33, 40), (4099, 64, 24), (9, 3001, 16), (300, 4096, 8)]


@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense(dtype, size, order):
    M, K, N = size
    d = Draw(M + 31 * K + 7 * N, dtype)
    x, w, b, res = d.rows(M, K), d.weight(K, N, order), d.vector(N), d.rows(M, N)
    y, intact = guarded(M, N, dtype)
    P.dense(x, w, out=y)
    O.check(y, O.dense(x, w, None, 0, None, None, dtype)[0], "product")
    assert intact()
    drop = (0.3, rng())
    y, pre = P.dense(x, w, b, act=P.ACT_GELU, dropout=drop, residual=res, pre=True)
    want, want_pre = O.dense(x, w, b, 2, (0.3, (KEY, STEP)), res, dtype)
    O.check(pre, want_pre, "pre")
    O.check(y, want, "y")


@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_RELU, P.ACT_GELU, P.ACT_SILU])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_epilogue(dtype, act):
    # every part of the epilogue by itself and with the others; wide values
    for i, (bias, p, residual) in enumerate(itertools.product((False, True), (0.0, 0.25, 1.0), (False, True))):
        for M, K, N in ((5, 40, 36), (150, 72, 131)):
            d = Draw(100 + i, dtype)
            x, w = d.rows(M, K, scale=4.0), d.weight(K, N, "io")
            b, res = d.vector(N) if bias else None, d.rows(M, N) if residual else None
            y = P.dense(x, w, b, act=act, dropout=(p, rng()) if p else None, residual=res)
            want = O.dense(x, w, b, act, (p, (KEY, STEP)) if p else None, res, dtype)[0]
            O.check(y, want, "%s p=%g residual=%s" % (bias, p, residual))


# row padding and an offset of the first element: alignment of 2 to 16 bytes
@pytest.mark.parametrize("pad,offset", [(0, 1), (8, 0), (8, 8), (1, 0), (3, 2), (4, 4), (6, 5)])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_strides(dtype, pad, offset):
    for M, K, N, order in ((37, 80, 72, "io"), (261, 136, 264, "oi"), (2, 264, 96, "io")):
        d = Draw(5, dtype)
        x, res = d.rows(M, K, pad, offset=offset), d.rows(M, N, pad, offset=offset)
        w = d.rows(K, N, pad, K ** -0.5, offset=offset) if order == "io" else \
            d.rows(N, K, pad, K ** -0.5, offset=offset).t()
        y, intact = guarded(M, N, dtype, pad)
        pre, intact_pre = guarded(M, N, dtype, offset)
        P.dense(x, w, act=P.ACT_SILU, residual=res, out=y, pre=pre)
        want, want_pre = O.dense(x, w, None, 3, None, res, dtype)
        O.check(y, want)
        O.check(pre, want_pre)
        assert intact() and intact_pre()
        dy = d.rows(M, N, pad, offset=offset)
        dx, intact = guarded(M, K, dtype, pad)
        grads = P.dense_backward(dy, x, w, pre=pre, act=P.ACT_SILU, dx=dx)
        for got, want, name in zip(grads, O.dense_backward(dy, x, w, pre, 3, None, dtype), ("dx", "dw", "db")):
            O.check(got, want, name)
        assert intact()
        assert grads[1].stride() == (torch.empty(K, N) if order == "io" else torch.empty(N, K).t()).stride()


@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_backward(dtype, size, order):
    M, K, N = size
    d = Draw(M + 31 * K + 7 * N, dtype)
    x, w, dy, pre = d.rows(M, K), d.weight(K, N, order), d.rows(M, N), d.rows(M, N)
    for act, p in ((0, 0.0), (2, 0.0), (3, 0.4), (0, 0.4), (1, 1.0)):
        grads = P.dense_backward(dy, x, w, pre=pre, act=act, dropout=(p, rng()) if p else None)
        want = O.dense_backward(dy, x, w, pre, act, (p, (KEY, STEP)) if p else None, dtype)
        for got, v, name in zip(grads, want, ("dx", "dw", "db")):
            O.check(got, v, "%s act %d p %g" % (name, act, p))


def test_dense_backward_long_sums():
    # more rows than one workgroup sums; few and many weights
    for dtype, M, K, N in ((torch.float32, 70000, 40, 24), (torch.bfloat16, 50001, 64, 256)):
        d = Draw(1, dtype)
        x, w, dy, pre = d.rows(M, K), d.weight(K, N, "io"), d.rows(M, N), d.rows(M, N)
        grads = P.dense_backward(dy, x, w, pre=pre, act=P.ACT_SILU)
        for got, v, name in zip(grads, O.dense_backward(dy, x, w, pre, 3, None, dtype), ("dx", "dw", "db")):
            O.check(got, v, name)


def test_dense_backward_parts():
    d = Draw(2, torch.float32)
    x, w, dy = d.rows(40, 24), d.weight(24, 16, "io"), d.rows(40, 16)
    dx, dw, db = P.dense_backward(dy, x, w)
    assert torch.equal(P.dense_backward(dy, x, w, dweight=False, bias=False)[0], dx)
    assert torch.equal(P.dense_backward(dy, x, w, dx=False, bias=False)[0], dw)
    assert torch.equal(P.dense_backward(dy, x, w, dx=False, dweight=False)[0], db)


def test_dense_gradient_by_differences():
    # the loss sum(y c) along a direction of each input, by central differences of
    # the fp32 forward pass: they are good to h^2 and 1/h of its rounding
    d = Draw(3, torch.float32)
    M, K, N = 20, 24, 28
    x, w, b, c = d.rows(M, K), d.weight(K, N, "io"), d.vector(N), d.rows(M, N)
    drop = (0.2, rng())
    for act in (P.ACT_NONE, P.ACT_GELU, P.ACT_SILU):
        pre = P.dense(x, w, b, act=act, dropout=drop, pre=True)[1]
        grads = P.dense_backward(c, x, w, pre=pre, act=act, dropout=drop)

        def loss(x, w, b):
            return float((P.dense(x, w, b, act=act, dropout=drop).double() * c.double()).sum())
        h = 2.0 ** -6
        for i, g in enumerate(grads):
            v = [x, w, b]
            t = torch.sign(g) + (g == 0)
            v[i] = v[i] + h * t
            up = loss(*v)
            v = [x, w, b]
            v[i] = v[i] - h * t
            down = loss(*v)
            exact = float((g.double() * t.double()).sum())
            assert abs((up - down) / (2 * h) - exact) <= 0.02 * abs(exact) + 0.05, (act, i)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_not_finite(dtype):
    # infinities and NaN reach the rows and columns that they belong to, and no
    # others; dropped ones nothing; the lowest value and sums beyond the type do
    # what 32-bit sums do
    M, K, N = 70, 96, 80
    d = Draw(4, dtype)
    x, w, res = d.rows(M, K), d.weight(K, N, "io"), d.rows(M, N)
    x[3, 5] = float("inf")
    x[10, 0] = float("nan")
    x[20] = torch.finfo(dtype).min
    w[7, 11] = float("-inf")
    y = P.dense(x, w, residual=res)
    bad = ~torch.isfinite(x).all(1)[:, None] | ~torch.isfinite(w).all(0)[None, :]
    v, e = O.dense(x, w, None, 0, None, res, dtype)[0]
    got = y.detach().cpu().double()
    ok = ~bad.cpu()
    ok[20] = False
    assert torch.isfinite(got[ok]).all()
    assert float(((got - v).abs() - e)[ok].max()) <= 0
    assert not torch.isfinite(got[bad.cpu()]).any()
    for r in (3, 10):
        assert torch.equal(torch.isnan(got[r]), torch.isnan(v[r]))
    # all dropped: the residual alone
    y = P.dense(x, w, dropout=(1.0, rng()), residual=res)
    assert torch.equal(y, res)
    g = P.dense_backward(y * float("inf"), x, w, dropout=(1.0, rng()), bias=True)
    assert (g[2] == 0).all()


def test_dense_smallest_values():
    # fp32 products keep their bits down to small operands
    d = Draw(6, torch.float32)
    for scale in (2.0 ** -60, 2.0 ** 50):
        x, w = d.rows(140, 64, scale=scale), d.weight(64, 136, "io")
        O.check(P.dense(x, w), O.dense(x, w, None, 0, None, None, torch.float32)[0])


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_no_rows(dtype):
    d = Draw(7, dtype)
    x, w = d.rows(0, 16), d.weight(16, 8, "io")
    assert P.dense(x, w).shape == (0, 8)
    dx, dw, db = P.dense_backward(d.rows(0, 8), x, w)
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    y, mean, rstd = P.layer_norm(x)
    assert y.shape == (0, 16) and mean.shape == rstd.shape == (0,)
    dx, dw, db = P.layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    assert P.dropout(x, 0.5, rng()).shape == (0, 16)


NORM_SIZES = [(1, 1), (1, 64), (2, 3), (1, 4096), (5, 77), (300, 128), (33, 129), (1000, 96), (64, 1000),
              (7, 2048), (9, 8192), (3, 10007), (2, 40000), (2049, 256), (70001, 8)]


@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("size", NORM_SIZES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_layer_norm(dtype, size, pad):
    rows, n = size
    d = Draw(rows + n, dtype)
    x = d.rows(rows, n, pad, 1.5, 0.7)
    w, b = d.vector(n, 0.3, 1.0), d.vector(n)
    y, intact = guarded(rows, n, dtype, pad)
    got = P.layer_norm(x, w, b, out=y)
    want = O.layer_norm(x, w, b, 1e-5, dtype)
    for g, v, name in zip(got, want, ("y", "mean", "rstd")):
        O.check(g, v, name)
    assert intact()
    O.check(P.layer_norm(x, None, b)[0], O.layer_norm(x, None, b, 1e-5, dtype)[0])
    O.check(P.layer_norm(x, w, None)[0], O.layer_norm(x, w, None, 1e-5, dtype)[0])
    x = x.clone()
    plain = P.layer_norm(x)[0]
    assert torch.equal(P.layer_norm(x, out=x)[0], plain)  # in place


@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("size", NORM_SIZES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_layer_norm_backward(dtype, size, pad):
    rows, n = size
    d = Draw(rows + n, dtype)
    x, dy, res = d.rows(rows, n, pad, 1.5, 0.7), d.rows(rows, n, pad), d.rows(rows, n, pad)
    w = d.vector(n, 0.3, 1.0)
    mean = x.float().mean(1)
    rstd = (x.float().var(1, unbiased=False) + 1e-5).rsqrt()
    dx, intact = guarded(rows, n, dtype, pad)
    got = P.layer_norm_backward(dy, x, mean, rstd, w, dresidual=res, dx=dx)
    for g, v, name in zip(got, O.layer_norm_backward(dy, x, mean, rstd, w, res, dtype), ("dx", "dw", "db")):
        O.check(g, v, name)
    assert intact()
    got = P.layer_norm_backward(dy, x, mean, rstd, None)
    for g, v, name in zip(got, O.layer_norm_backward(dy, x, mean, rstd, None, None, dtype), ("dx", "dw", "db")):
        O.check(g, v, name)
    alone = P.layer_norm_backward(dy, x, mean, rstd, params=False)
    assert torch.equal(alone, got[0])
    dy = dy.clone()
    again = P.layer_norm_backward(dy, x, mean, rstd, dx=dy)  # in place
    assert all(torch.equal(a, b) for a, b in zip(again, got))


def test_layer_norm_values():
    # a row of one value: variance 0; values far from 0 with a small spread;
    # infinities and NaN stay in their rows
    x = torch.full((4, 64), 3.0, device="cuda:0")
    x[1] = 1000.0 + torch.arange(64, device="cuda:0") / 64
    x[2, 5] = float("nan")
    x[3, 6] = float("inf")
    y, mean, rstd = P.layer_norm(x)
    assert (y[0] == 0).all() and mean[0] == 3.0
    O.check(y[1:2], O.layer_norm(x[1:2], None, None, 1e-5, torch.float32)[0])
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[3]).any()


def test_layer_norm_gradient_by_differences():
    d = Draw(8, torch.float32)
    x, w, b, c = d.rows(6, 40), d.vector(40, 0.3, 1.0), d.vector(40), d.rows(6, 40)
    _, mean, rstd = P.layer_norm(x, w, b)
    grads = P.layer_norm_backward(c, x, mean, rstd, w)

    def loss(x, w, b):
        return float((P.layer_norm(x, w, b)[0].double() * c.double()).sum())
    h = 2.0 ** -7
    for i, g in enumerate(grads):
        t = torch.sign(g) + (g == 0)
        up, down = [x, w, b], [x, w, b]
        up[i], down[i] = up[i] + h * t, down[i] - h * t
        exact = float((g.double() * t.double()).sum())
        assert abs((loss(*up) - loss(*down)) / (2 * h) - exact) <= 0.02 * abs(exact) + 0.05, i


@pytest.mark.parametrize("size,pad", [((1, 1), 0), ((1, 4096), 0), ((3, 7), 2), ((1001, 77), 3), ((64, 1024), 0),
                                      ((33, 130), 6), ((5, 3000), 1), ((2048, 96), 32)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dropout(dtype, size, pad):
    rows, n = size
    d = Draw(rows + n, dtype)
    x, res = d.rows(rows, n, pad), d.rows(rows, n, pad)
    for p in (0.0, 0.1, 0.5, 0.999, 1.0):
        for key, step in ((KEY, STEP), (-1, 2 ** 32 + 5), (0, 0)):
            y, intact = guarded(rows, n, dtype, pad)
            P.dropout(x, p, rng(key, step), residual=res, out=y)
            drop = (p, (key & (2 ** 64 - 1), step))
            O.check(y, O.dropout(x, drop, res, dtype))
            assert intact()
    y = P.dropout(x, 0.5, rng())
    O.check(y, O.dropout(x, (0.5, (KEY, STEP)), None, dtype))
    a, b = x.clone(), res.clone()
    want = P.dropout(x, 0.5, rng(), residual=res)
    assert torch.equal(P.dropout(a, 0.5, rng(), residual=res, out=a), want)
    assert torch.equal(P.dropout(x, 0.5, rng(), residual=b, out=b), want)


def test_dropout_masked_values():
    # a dropped element is zero whatever it was
    x = torch.full((64, 64), float("nan"), device="cuda:0")
    keep = torch.from_numpy(O.philox_words(KEY, STEP, 64, 64) >= 2 ** 31).to("cuda:0")
    x[keep] = 1.0
    y = P.dropout(x, 0.5, rng())
    assert torch.equal(y, keep.float() * 2)
    x[~keep] = float("inf")
    assert torch.equal(P.dropout(x, 0.5, rng()), keep.float() * 2)


def test_dense_draws_the_mask_of_dropout():
    d = Draw(9, torch.float32)
    x, w = d.rows(45, 32), d.weight(32, 77, "io")
    y = P.dense(x, w)
    assert torch.equal(P.dense(x, w, dropout=(0.35, rng())), P.dropout(y, 0.35, rng()))


def test_same_bits_and_other_streams():
    # repeated calls, calls on another stream and through plans give the same bits
    d = Draw(10, torch.bfloat16)
    x, w, b, dy, pre = d.rows(500, 256), d.weight(256, 384, "io"), d.vector(384), d.rows(500, 384), d.rows(500, 384)
    drop = (0.1, rng())
    mean, rstd = P.layer_norm(x)[1:]

    def calls(stream=None):
        return (P.dense(x, w, b, act=P.ACT_GELU, dropout=drop, stream=stream),
                *P.dense_backward(dy, x, w, pre=pre, act=P.ACT_GELU, dropout=drop, stream=stream),
                *P.layer_norm(x, stream=stream), *P.layer_norm_backward(x, x, mean, rstd, stream=stream),
                P.dropout(x, 0.1, drop[1], stream=stream))
    first = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = calls(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(first, other):
        assert torch.equal(a, c)
    plan = P.dense_backward_plan(dy, x, w, pre=pre, act=P.ACT_GELU, dropout=drop)
    for _ in range(3):
        for a, c in zip(plan(), first[1:4]):
            assert torch.equal(a, c)


def test_graph_replays():
    # captured, with new inputs and a new mask between the replays
    d = Draw(11, torch.bfloat16)
    x, w, b = d.rows(300, 128), d.weight(128, 256, "io"), d.vector(256)
    dy, r = d.rows(300, 256), rng()
    nw, nb = d.vector(128), d.vector(128)

    def step():
        h, mean, rstd = P.layer_norm(x, nw, nb)
        y, pre = P.dense(h, w, b, act=P.ACT_SILU, dropout=(0.2, r), pre=True)
        dh, dw, db = P.dense_backward(dy, h, w, pre=pre, act=P.ACT_SILU, dropout=(0.2, r))
        return (y, dw, db, *P.layer_norm_backward(dh, x, mean, rstd, nw, dresidual=x),
                P.dropout(y, 0.3, r))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for rep in range(4):
        x.mul_(1.25)
        r[1] += 1
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(outs, eager):
            assert torch.equal(a, c), rep


def test_leading_axes():
    # rows are all leading axes; a multivector tensor's channels and blades are features
    d = Draw(12, torch.float32)
    x = d.rows(6 * 5, 32).view(6, 5, 32)
    w = d.weight(32, 12, "io")
    assert torch.equal(P.dense(x, w), P.dense(x.view(30, 32), w).view(6, 5, 12))
    assert torch.equal(P.layer_norm(x[:, 2])[0], P.layer_norm(x[:, 2].contiguous())[0])
    mv = d.rows(10, 32).view(10, 8, 4)
    y, _, _ = P.layer_norm(mv.flatten(1))
    assert y.shape == (10, 32)
    assert P.dense(x[0, 0], w).shape == (12,)


# many rows and a short contraction: the panel kernel (rows from 16384, K up to 128)
@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", [(16384, 128, 128), (16385, 64, 300), (20001, 100, 129), (16400, 13, 520), (40003, 17, 8),
                                  (17000, 128, 1), (33333, 8, 257)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_short_contraction(dtype, size, order):
    M, K, N = size
    d = Draw(M + K + N, dtype)
    x, w, b, res = d.rows(M, K, 3), d.weight(K, N, order), d.vector(N), d.rows(M, N)
    y, intact = guarded(M, N, dtype)
    got, pre = P.dense(x, w, b, act=P.ACT_SILU, dropout=(0.2, rng()), residual=res, pre=True, out=y)
    want, want_pre = O.dense(x, w, b, 3, (0.2, (KEY, STEP)), res, dtype)
    O.check(pre, want_pre, "pre")
    O.check(got, want, "y")
    assert intact()


@pytest.mark.parametrize("M,K,N", [(5, 96, 80), (40, 520, 48), (16390, 112, 80), (300, 640, 80)])
def test_dense_not_finite_paths(M, K, N):
    # fp32 by every kernel: few rows, panels, tiles (split contraction too):
    # infinities stay in their rows and columns, and values that bf16 parts
    # cannot hold come out as fp32 products give them
    d = Draw(14, torch.float32)
    x, w = d.rows(M, K), d.weight(K, N, "io")
    x[2, 3] = float("inf")
    x[3] = 0.0
    x[3, 1] = 3e38
    w[5, 7] = float("nan")
    w[1, 9] = 2.0 ** -126
    y = P.dense(x, w).cpu().double()
    v, e = O.dense(x, w, None, 0, None, None, torch.float32)[0]
    good = torch.isfinite(v)
    big = v.abs() > 3.4e38
    assert torch.equal(torch.isnan(y), torch.isnan(v))
    assert not torch.isfinite(y[~good]).any() and (y[big & good].abs() > 3e38).all()
    assert float(((y - v).abs() - e)[good & ~big].max()) <= 0


def test_dense_split_contraction():
    # few outputs and a long contraction: parts joined in order, the epilogue in the join
    for dtype in DTYPES:
        d = Draw(15, dtype)
        for M, K, N, order in ((96, 8192, 72, "io"), (130, 5003, 61, "oi"), (72, 4096, 256, "oi")):
            x, w, b, res = d.rows(M, K), d.weight(K, N, order), d.vector(N), d.rows(M, N)
            y, intact = guarded(M, N, dtype)
            P.dense(x, w, b, act=P.ACT_GELU, dropout=(0.15, rng()), residual=res, out=y)
            O.check(y, O.dense(x, w, b, 2, (0.15, (KEY, STEP)), res, dtype)[0], str((M, K, N)))
            assert intact()
            again = P.dense(x, w, b, act=P.ACT_GELU, dropout=(0.15, rng()), residual=res)
            assert torch.equal(again, y)


def test_dense_large_tiles():
    # 256 x 256 tiles with ragged edges, both orders, and their gradient
    for dtype in (torch.bfloat16, torch.float16):
        d = Draw(16, dtype)
        M, K, N = 2100, 1096, 2008
        for order in ("io", "oi"):
            x, w, b = d.rows(M, K), d.weight(K, N, order), d.vector(N)
            O.check(P.dense(x, w, b, act=P.ACT_RELU), O.dense(x, w, b, 1, None, None, dtype)[0], order)
            dy = d.rows(M, N)
            for got, v, name in zip(P.dense_backward(dy, x, w), O.dense_backward(dy, x, w, None, 0, None, dtype),
                                    ("dx", "dw", "db")):
                O.check(got, v, name)


def test_dense_in_place_residual():
    # y may be the residual, by every kernel
    for M, K, N in ((3, 64, 72), (200, 96, 264), (100, 4096, 40), (16400, 64, 96)):
        d = Draw(17, torch.bfloat16)
        x, w, res = d.rows(M, K), d.weight(K, N, "io"), d.rows(M, N)
        want = P.dense(x, w, residual=res)
        assert torch.equal(P.dense(x, w, residual=res, out=res), want)


def test_activations_over_the_range():
    # values and slopes at every fp32 exponent that matters, at the ends too
    v = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([-100.0, 100.0, -3e38, 3e38, 0.0, -0.0, 1e-30, -1e-30])])
    x = v.to("cuda:0")[:, None]
    one = torch.ones(1, 1, device="cuda:0")
    for act in (P.ACT_RELU, P.ACT_GELU, P.ACT_SILU):
        y = P.dense(x, one, act=act).cpu().double()[:, 0]
        want = O.act(act, v.double())
        # 16 roundings of the value, and of the value's size near zero
        assert float(((y - want).abs() - 2.0 ** -20 * want.abs() - 1e-37)[v > -12.1].max()) <= 0, act
        assert torch.isfinite(y).all()
        g = P.dense_backward(torch.ones_like(x), x, one, pre=x, act=act)[0].cpu().double()[:, 0]
        want = O.slope(act, v.double())
        inside = v.abs() < 1e30
        assert float((g - want).abs()[inside].max()) <= 2.0 ** -20 * 2, act


# few rows past a long contraction: whole stages in rounds, a rest of rounds and
# of a stage, and 1 to 31 columns in the last workgroup; NaN beside the operands
@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", [(1, 520, 4096 + 5), (3, 8200, 4100), (16, 5003, 4106), (24, 4167, 4123), (50, 4101, 4097),
                                  (64, 2303, 2079), (7, 1024, 33), (31, 700, 15)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_few_rows(dtype, size, order):
    M, K, N = size
    d = Draw(M + K + N, dtype)
    x, w = d.rows(M, K), d.weight(K, N, order)

    def beside(t, pad):
        big = torch.full((t.shape[0] + 1, t.shape[1] + pad), float("nan"), dtype=dtype, device="cuda:0")
        big[:-1, :t.shape[1]] = t
        return big[:-1, :t.shape[1]]
    xs = beside(x, 5)
    ws = beside(w, 3) if order == "io" else beside(w.t(), 3).t()
    b, res = d.vector(N), d.rows(M, N)
    drop = (0.25, rng())
    want, want_pre = O.dense(x, w, b, 1, (0.25, (KEY, STEP)), res, dtype)
    for left, right in ((x, w), (xs, ws)):
        y, intact = guarded(M, N, dtype)
        got, pre = P.dense(left, right, b, act=P.ACT_RELU, dropout=drop, residual=res, pre=True, out=y)
        O.check(pre, want_pre, "pre")
        O.check(got, want, "y")
        assert intact()


def test_joins_of_many_outputs():
    # the two joins of split contractions, groups of four columns that end inside
    for dtype in DTYPES:
        d = Draw(18, dtype)
        for M, K, N in ((1003, 1531, 777), (130, 4099, 250), (1001, 1601, 1022)):
            x, w, b, res = d.rows(M, K), d.weight(K, N, "io"), d.vector(N), d.rows(M, N)
            y, intact = guarded(M, N, dtype)
            P.dense(x, w, b, act=P.ACT_SILU, dropout=(0.15, rng()), residual=res, out=y)
            O.check(y, O.dense(x, w, b, 3, (0.15, (KEY, STEP)), res, dtype)[0], str((M, K, N)))
            assert intact()
