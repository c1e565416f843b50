"""Edges of the feed-forward operators on the GPU, against the plain
implementations in 64 bits of ff_oracle.py (which derives the bounds)."""
import pytest
import torch

import ff_oracle as O
import paper_2507_01040_amd as P
from ff_cases import LARGE_TILES
from test_feed_forward_gpu import DTYPES, KEY, STEP, Draw, guarded, ids, rng

pytestmark = pytest.mark.gpu


def _guarded_weight(order, K, N, dtype, pad):
    view, intact = guarded(N, K, dtype, pad) if order == "oi" else guarded(K, N, dtype, pad)
    return (view.t() if order == "oi" else view), intact


@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", [(40, 1, 512), (40, 512, 1), (3, 1, 1), (200, 1, 2), (70, 24, 36)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_weight_gradient_stays_in_its_tensor(dtype, size, order):
    # one input or output feature, padded weights and gradients, everything around them
    M, K, N = size
    d = Draw(M + K + N, dtype)
    x, dy = d.rows(M, K), d.rows(M, N)
    w = _guarded_weight(order, K, N, dtype, 6)[0]
    w.copy_(d.weight(K, N, order))
    want = O.dense_backward(dy, x, w, None, 0, None, dtype)
    for pad in (None, 0, 3):
        dw, intact = _guarded_weight(order, K, N, dtype, pad) if pad is not None else (None, lambda: True)
        db, intact_b = guarded(1, N, dtype, 5)
        got = P.dense_backward(dy, x, w, dweight=dw, dbias=db[0])
        for g, v, name in zip(got, want, ("dx", "dw", "db")):
            O.check(g, v, "%s pad %s" % (name, pad))
        assert intact() and intact_b()


def test_buffers_of_a_call_on_another_stream():
    # a block that the current stream has just freed, perhaps with readers still
    # queued there, is not what a call on another stream writes
    d = Draw(1, torch.float32)
    x, w, dy = d.rows(300, 256), d.weight(256, 256, "io"), d.rows(300, 256)
    mean, rstd = P.layer_norm(x)[1:]
    side = torch.cuda.Stream()
    drop = (0.5, rng())
    calls = [lambda s: (P.dense(x, w, stream=s),), lambda s: P.dense_backward(dy, x, w, stream=s),
             lambda s: P.layer_norm(x, stream=s), lambda s: P.layer_norm_backward(dy, x, mean, rstd, stream=s),
             lambda s: (P.dropout(x, *drop, stream=s),)]
    for i, call in enumerate(calls):
        want = call(None)
        torch.cuda.synchronize()
        freed = [torch.empty_like(t) for t in want for _ in range(4)]
        places = {t.data_ptr() for t in freed}
        del freed
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        assert not places & {t.data_ptr() for t in got}, i
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    # by a raw handle, through a plan
    plan = P.dense_plan(x, w)
    want = plan().clone()
    plan.out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = plan(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


# each kernel of the dense layer: few rows, tiles, panels, a split contraction
@pytest.mark.parametrize("M,K,N", [(3, 64, 72), (200, 96, 136), (16400, 64, 40), (72, 4096, 40)])
@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_RELU, P.ACT_GELU, P.ACT_SILU])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_nan_passes_the_activations(dtype, act, M, K, N):
    # a NaN in a row of x stays in that row of y, whatever the activation; so does
    # one of the pre-activations in the gradient, where its element is kept
    d = Draw(21, dtype)
    x, w, res = d.rows(M, K), d.weight(K, N, "io"), d.rows(M, N)
    x[2, K - 1] = float("nan")
    y, pre = P.dense(x, w, act=act, residual=res, pre=True)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda:0")
    bad[2] = True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(torch.isnan(pre), bad)
    if act == P.ACT_NONE:
        return
    x[2, K - 1] = 0.0
    pre = d.rows(M, N)
    pre[2, 5] = float("nan")
    keep = torch.from_numpy(O.philox_words(KEY, STEP, 3, 8)[2, 5:6] >= 2 ** 31).to("cuda:0")
    for drop, kept in ((None, True), ((0.5, rng()), bool(keep))):
        dx, dw, db = P.dense_backward(res, x, w, pre=pre, act=act, dropout=drop)
        row, col = torch.zeros(M, dtype=torch.bool, device="cuda:0"), torch.zeros(N, dtype=torch.bool, device="cuda:0")
        row[2], col[5] = kept, kept
        assert torch.equal(torch.isnan(dx), row[:, None].expand(M, K))
        assert torch.equal(torch.isnan(dw), col[None, :].expand(K, N))
        assert torch.equal(torch.isnan(db), col)


def test_relu_values():
    v = torch.tensor([-0.0, 0.0, 1e-40, -1e-40, 3e38, -3e38, float("inf"), float("-inf"), float("nan")], device="cuda:0")
    one = torch.ones(1, 1, device="cuda:0")
    y = P.dense(v[:, None], one, act=P.ACT_RELU)[:, 0]
    assert torch.equal(y[:-1], torch.tensor([0.0, 0.0, 1e-40, 0.0, 3e38, 0.0, float("inf"), 0.0], device="cuda:0"))
    assert torch.isnan(y[-1])
    g = P.dense_backward(torch.ones_like(v)[:, None], v[:, None], one, pre=v[:, None], act=P.ACT_RELU)[0][:, 0]
    assert g[:-1].tolist() == [0.0, 0.0, 1.0, 0.0, 1.0, 0.0, 1.0, 0.0] and torch.isnan(g[-1])


def _exact_gradient(dy, x, w, pre, act, dropout, dtype):
    """((dx, bound), (dw, bound), (db, bound)) where g is rounded nowhere: fp32 sums
    of exact products, the scale and one rounding to the type (bounds as in
    ff_oracle.py)."""
    dy, x, w = (v.detach().cpu().double() for v in (dy, x, w))
    M, N = dy.shape
    g = dy if not act else dy * O.slope(act, pre.detach().cpu().double())
    if dropout is not None:
        g = g * O.mask(dropout, M, N)
    u, t = O.UNIT[dtype], O.TINY[dtype]

    def out(v, size, n):
        e = (O.LAMBDA * n ** 0.5 + O.COST) * O.U * size
        return v, e * (1 + u) + 2 * u * v.abs() + t
    return (out(g @ w.t(), g.abs() @ w.abs().t(), N), out(x.t() @ g, x.abs().t() @ g.abs(), M),
            out(g.sum(0), g.abs().sum(0), M))


@pytest.mark.parametrize("size", [(40, 64, 520), (300, 512, 256), (16400, 40, 96)], ids=str)
@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_RELU])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=ids)
def test_gradient_without_rounding(dtype, act, size):
    # a dropped layer without an activation or with ReLU: g is dy or zero, and the
    # dropout's 1 / (1 - p), no value of the type, multiplies the fp32 sums
    M, K, N = size
    d = Draw(M + N, dtype)
    x, w, dy, pre = d.rows(M, K), d.weight(K, N, "io"), d.rows(M, N), d.rows(M, N)
    got = P.dense_backward(dy, x, w, pre=pre, act=act, dropout=(0.3, rng()))
    for g, v, name in zip(got, _exact_gradient(dy, x, w, pre, act, (0.3, (KEY, STEP)), dtype), ("dx", "dw", "db")):
        O.check(g, v, name)


@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_RELU, P.ACT_GELU, P.ACT_SILU])
def test_fp16_gradient_of_large_values(act):
    # output gradients up to fp16's largest value: dx and dw are far below it, and
    # finite, though dy f'(pre) / (1 - p) is not an fp16 value
    M, K, N = 70, 48, 80
    d = Draw(22, torch.float16)
    x, w = d.rows(M, K, scale=1e-3), d.weight(K, N, "io") * 0.01
    dy = torch.where(d.rows(M, N) > 0, 65504.0, -65504.0).half()
    pre = d.rows(M, N, scale=0.1, shift=1.5)  # about the steepest point of GELU
    for p in (0.0, 0.6):
        drop = (p, (KEY, STEP)) if p else None
        dx, dw, db = P.dense_backward(dy, x, w, pre=pre, act=act, dropout=(p, rng()) if p else None)
        want = O.dense_backward(dy, x, w, pre, act, drop, torch.float16)
        assert float(want[0][0].abs().max()) < 65504 and float(want[1][0].abs().max()) < 65504
        O.check(dx, want[0], "dx p %g" % p)
        O.check(dw, want[1], "dw p %g" % p)


def test_silu_keeps_the_digits_of_its_left_tail():
    # e = exp(-|v|), 1 + e, its reciprocal and three products round to about 8 units
    # of 2^-24 of the value (16 allowed); the slope's 1 + v (1 - s) adds as many times
    # |v| (1 - s) / |1 + v (1 - s)|, at most 2.4 from v = -2 on (32 allowed).  Results
    # below the smallest normal float are multiples of 2^-149.
    v = torch.cat([torch.linspace(-104, 12, 8001), torch.linspace(-89, -86, 2000)])
    x = v.to("cuda:0")[:, None]
    one = torch.ones(1, 1, device="cuda:0")
    y = P.dense(x, one, act=P.ACT_SILU).cpu().double()[:, 0]
    want = O.act(3, v.double())
    assert float(((y - want).abs() - 2.0 ** -20 * want.abs() - 110 * 2.0 ** -149).max()) <= 0
    g = P.dense_backward(torch.ones_like(x), x, one, pre=x, act=P.ACT_SILU)[0].cpu().double()[:, 0]
    want = O.slope(3, v.double())
    tail = v <= -2
    assert float(((g - want).abs() - 2.0 ** -19 * want.abs() - 110 * 2.0 ** -149)[tail].max()) <= 0
    assert float((g - want).abs()[~tail].max()) <= 2.0 ** -19


def test_grids_of_several_rows():
    # more workgroups than one row of a grid holds: every output written, and right
    for dtype, M, K, N in ((torch.bfloat16, 1, 1, (1 << 23) + 130), (torch.float32, (1 << 23) + 1, 2, 1),
                           (torch.float16, (1 << 23) + 129, 1, 2)):
        d = Draw(M + N, dtype)
        x, w = torch.ones(M, K, dtype=dtype, device="cuda:0"), torch.ones(K, N, dtype=dtype, device="cuda:0")
        (x if M > 1 else w).copy_(torch.arange(max(M, N), device="cuda:0").remainder(251).view(-1, 1) if M > 1 else
                                  torch.arange(N, device="cuda:0").remainder(251).view(1, -1))
        y = torch.full((M, N), -1.0, dtype=dtype, device="cuda:0")
        P.dense(x, w, d.vector(N) * 0, out=y)
        assert torch.equal(y, x.sum(1, keepdim=True) * w.sum(0, keepdim=True) / K)
    x = torch.arange((1 << 25) + 9, device="cuda:0", dtype=torch.float32).remainder_(8191).expand(9, -1)
    x = x + torch.arange(9, device="cuda:0")[:, None]
    y = P.dropout(x, 0.0, rng(), residual=x)
    assert torch.equal(y, x + x)


@pytest.mark.parametrize("dtype,order", [(torch.bfloat16, "io"), (torch.bfloat16, "oi"), (torch.float16, "io"),
                                         (torch.float16, "oi")], ids=ids)
def test_large_tiles(dtype, order):
    # the 256 x 256 tiles (test_feed_forward_on_cpu.py asserts that these sizes take
    # them): ragged edges, a last stage that is not whole, two stages, split
    # contractions, the whole epilogue
    for i, ((M, K, N), _, backward) in enumerate(LARGE_TILES):
        if backward and (dtype == torch.bfloat16) != (order == "io") and i == 3:
            continue  # (the oracle's time)
        d = Draw(M + K + N, dtype)
        x, w, b, res = d.rows(M, K, 8), d.weight(K, N, order), d.vector(N), d.rows(M, N, 3)
        y, intact = guarded(M, N, dtype)
        got, pre = P.dense(x, w, b, act=P.ACT_GELU, dropout=(0.15, rng()), residual=res, pre=True, out=y)
        want, want_pre = O.dense(x, w, b, 2, (0.15, (KEY, STEP)), res, dtype)
        O.check(pre, want_pre, "pre %d" % i)
        O.check(got, want, "y %d" % i)
        assert intact()
        if backward:
            dy = d.rows(M, N)
            dx, intact = guarded(M, K, dtype)
            dw, intact_w = _guarded_weight(order, K, N, dtype, 5)
            got = P.dense_backward(dy, x, w, pre=pre, act=P.ACT_RELU, dx=dx, dweight=dw)
            for g, v, name in zip(got, O.dense_backward(dy, x, w, pre, 1, None, dtype), ("dx", "dw", "db")):
                O.check(g, v, "%s %d" % (name, i))
            assert intact() and intact_w()
