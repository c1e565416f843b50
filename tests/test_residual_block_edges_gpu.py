"""What calls of the 8-bit operators and the block norm share with the other operators:
graphs, streams, the same bits, no rows, leading axes, NaN in its place, precision."""
import pytest
import torch

import block_oracle as B
import ff_oracle as O
import paper_2507_01040_amd as P
from test_feed_forward_gpu import DTYPES, ids, rng
from test_residual_block_gpu import Eight

pytestmark = pytest.mark.gpu


def _step(v, M=300, K=192, N=520, dtype=torch.bfloat16):
    """A step of a block, forward, served and backward, on tensors that stay."""
    x, r, w1, w2 = v.rows(M, K), v.rows(M, K), v.weight(K, N, "oi"), v.weight(N, K, "oi")
    b1, g, n = v.vector(N), v.rows(3, K), v.vector(K)
    drop = (0.25, rng())
    state = [x, r, drop[1]]

    def step(stream=None):
        k = dict(stream=stream)
        h = P.quantize(x, **k)
        s1, s2 = P.quantize(w1.t(), **k), P.quantize(w2.t(), **k)
        a = P.dense_int8(*h, s1[0].t(), s1[1], b1, act=P.ACT_SILU, **k)
        y = P.dense_int8(*P.quantize(a, **k), s2[0].t(), s2[1], residual=r, **k)
        out, normed, stats = P.block_norm(y, r, gate=g, weight=n, bias=n, next_weight=n, **k)
        grads = P.block_norm_backward(r, x, y, out, stats, gate=g, weight=n, bias=n, next_weight=n, **k)
        pre = P.quantize(a, group=128, **k)
        more = P.dense_backward_int8(grads.dx, *P.quantize(a, group=128, **k), w2, **k)
        last = P.dense_backward_int8(more[0], *h, w1, *pre, act=P.ACT_GELU, dropout=drop, **k)
        values = P.dequantize(*pre, dtype=dtype, **k)
        return [*h, a, y, out, normed, stats, *(t for t in grads if t is not None), *more, *last, values]
    return step, state


def test_same_bits_and_other_streams():
    for dtype in (torch.bfloat16, torch.float16):
        step, _ = _step(Eight(31, dtype), dtype=dtype)
        want = step()
        for a, b in zip(step(), want):
            assert torch.equal(a, b)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = step(side)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_graph_replays():
    step, (x, r, random) = _step(Eight(32, torch.bfloat16))
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
        random[1] += 1
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, c) in enumerate(zip(outs, eager)):
            assert torch.equal(a, c), (rep, i)


def test_two_graphs_have_workspaces_of_their_own():
    # two captured gradients, replayed one after the other and then together
    v = Eight(33, torch.bfloat16)
    M, K, N = 700, 512, 640
    w, calls, kept = v.weight(K, N, "io"), [], []  # (a plan's buffers live as long as it does)
    for _ in range(2):
        x, dy = P.quantize(v.rows(M, K), group=128), v.rows(M, N)
        pre = P.quantize(v.rows(M, N), group=128)
        plan = P.dense_backward_int8_plan(dy, *x, w, *pre, act=P.ACT_GELU)
        n = P.block_norm_backward_plan(dy, None, dy, None, torch.ones(4, M, device="cuda:0"), weight=v.vector(N))
        want = [t.clone() for t in (*plan(), *(t for t in n() if t is not None))]
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph):
            plan(torch.cuda.current_stream())
            n(torch.cuda.current_stream())
        kept.append((plan, n))
        calls.append((graph, side, (*plan.out, *(t for t in n.out if t is not None)), want))
    torch.cuda.synchronize()
    for together in (False, True):
        for graph, side, outs, _ in calls:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        for graph, side, _, _ in calls:
            with torch.cuda.stream(side):
                graph.replay()
            if not together:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        for _, _, outs, want in calls:
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_no_rows(dtype):
    v = Eight(34, dtype)
    none, w = torch.empty(0, 200, dtype=dtype, device="cuda:0"), v.vector(200)
    q, s = P.quantize(none, group=128)
    assert q.shape == (0, 200) and s.shape == (0, 2) and P.dequantize(q, s).shape == (0, 200)
    q1, s1 = P.quantize(none)
    w8, ws = P.quantize(v.rows(5, 200))
    assert P.dense_int8(q1, s1, w8.t(), ws, dtype=dtype).shape == (0, 5)
    dy = torch.empty(0, 5, dtype=dtype, device="cuda:0")
    p8, ps = P.quantize(dy)
    dx, dw, db = P.dense_backward_int8(dy, q, s, v.weight(200, 5, "io"), p8, ps, act=P.ACT_GELU)
    assert dx.shape == (0, 200) and not dw.any() and not db.any()
    out, normed, stats = P.block_norm(none, none, gate=w, weight=w, next_weight=w)
    assert out.shape == normed.shape == (0, 200) and stats.shape == (4, 0)
    g = P.block_norm_backward(none, none, none, none, stats, gate=v.rows(3, 200), weight=w, bias=w, next_weight=w, next_bias=w)
    assert g.dgate.shape == (3, 200) and not any(t.any() for t in g[2:])


def test_leading_axes():
    v = Eight(35, torch.float32)
    x = v.rows(30, 192).view(6, 5, 192)
    q, s = P.quantize(x, group=128)
    assert q.shape == x.shape and s.shape == (30, 2) and torch.equal(q.view(30, 192), P.quantize(x.view(30, 192), group=128)[0])
    w, ws = P.quantize(v.rows(12, 192))
    q, s = P.quantize(x)
    assert P.dense_int8(q, s, w.t(), ws, dtype=torch.float32).shape == (6, 5, 12)
    assert P.quantize(x[0, 0])[1].shape == (1, 1) and P.dense_int8(q[0, 0], s[:1], w.t(), ws).dtype == torch.bfloat16
    out, normed, _ = P.block_norm(x, x, gate=v.rows(6, 192))
    flat = P.block_norm(x.view(30, 192), x.view(30, 192), gate=torch.zeros(1, 192, device="cuda:0"))
    assert out.shape == normed.shape == x.shape and flat[0].shape == (30, 192)
    with pytest.raises(ValueError, match="rows have no single stride"):
        P.quantize(v.rows(60, 192).view(6, 10, 192)[:, 1:6])


@pytest.mark.parametrize("size", [(5, 300, 40), (200, 256, 264), (70, 2048, 40)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_values_that_are_not_finite_stay_in_their_place(dtype, size):
    # an infinity of a row makes NaN of its row, of its group in the weight's gradient, and of
    # nothing else
    M, K, N = size
    v = Eight(36, dtype)
    x, w, dy, pre = v.rows(M, K), v.weight(K, N, "io"), v.rows(M, N), v.rows(M, N)
    x[2, 130] = float("inf")
    q, s = P.quantize(x)
    w8, ws = P.quantize(w.t().contiguous())
    y = P.dense_int8(q, s, w8.t(), ws, act=P.ACT_GELU, dtype=dtype)
    row = torch.zeros(M, 1, dtype=torch.bool, device="cuda:0")
    row[2] = True
    assert torch.equal(torch.isnan(y), row.expand(M, N))
    for act in (P.ACT_RELU, P.ACT_SILU):
        q, s = P.quantize(x, group=128)
        dx, dw, db = P.dense_backward_int8(dy, q, s, w, *P.quantize(pre, group=128), act=act)
        group = torch.zeros(K, 1, dtype=torch.bool, device="cuda:0")
        group[128:256] = True
        kept = dy[2] != 0 if act == P.ACT_SILU else torch.ones(N, dtype=torch.bool, device="cuda:0")
        assert bool(kept.all())
        assert torch.equal(torch.isnan(dw), group.expand(K, N)) and not torch.isnan(dx).any() and not torch.isnan(db).any()
        bad = pre.clone()
        bad[M - 1, N - 1] = float("nan")
        dx, dw, db = P.dense_backward_int8(dy, *P.quantize(x.nan_to_num(0, 0, 0), group=128), w, *P.quantize(bad, group=128), act=act)
        row = torch.zeros(M, 1, dtype=torch.bool, device="cuda:0")
        row[M - 1] = True
        col = torch.zeros(N, dtype=torch.bool, device="cuda:0")
        col[(N - 1) // 128 * 128:] = True
        assert torch.equal(torch.isnan(dx), row.expand(M, K))
        assert torch.equal(torch.isnan(db), col) and torch.equal(torch.isnan(dw), col.expand(K, N))
    h = v.rows(M, K)
    h[1, 7] = float("nan")
    out, normed, stats = P.block_norm(h, x.nan_to_num(0, 0, 0))
    row = torch.zeros(M, 1, dtype=torch.bool, device="cuda:0")
    row[1] = True
    assert torch.equal(torch.isnan(out), row.expand(M, K)) and torch.equal(torch.isnan(normed), row.expand(M, K))


@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_RELU, P.ACT_GELU, P.ACT_SILU])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=ids)
@pytest.mark.parametrize("size", [(2000, 256, 384), (1500, 300, 130)], ids=str)
def test_weight_gradient_has_one_rounded_operand(dtype, act, size):
    # 2-norm error over the result: the output's rounding and one operand's, each uniform
    # over half a step of a significand in [1, 2): at most u / 3^0.5 rms, so 2^0.5 u / 3^0.5 =
    # 0.82 u together; two rounded operands would make it 1.0 u where all three are at most
    # that, and measured significands are spread (a mean of 0.72 of it)
    M, K, N = size
    v = Eight(37, dtype)
    x, dy, pre = v.rows(M, K), v.rows(M, N, scale=0.05), v.rows(M, N)
    for order in ("io", "oi"):
        for group in (None, 128):
            q, p = P.quantize(x, group=group), P.quantize(pre, group=group)
            dw = P.dense_backward_int8(dy, *q, v.weight(K, N, order), *p, act=act, dx=False, bias=False)[0]
            want = B.values(*q).t() @ (dy.cpu().double() * O.slope(act, B.values(*p)))
            err = float((dw.cpu().double() - want).norm() / want.norm())
            assert err <= 0.82 * O.UNIT[dtype], err / O.UNIT[dtype]


def test_int8_in_place_residual():
    v = Eight(38, torch.float16)
    for M, K, N in ((3, 512, 72), (200, 96, 264), (100, 4096, 40), (300, 777, 130), (520, 1040, 512)):
        x, w, res = v.int8(M, K), v.int8(N, K), v.rows(M, N)
        xs, ws = v.scale(M), v.scale(N, size=1e-4)
        want = P.dense_int8(x, xs, w.t(), ws, residual=res)
        assert torch.equal(P.dense_int8(x, xs, w.t(), ws, residual=res, out=res), want)


def test_plans_on_a_raw_handle():
    v = Eight(39, torch.bfloat16)
    x, w = P.quantize(v.rows(40, 512)), P.quantize(v.rows(64, 512))
    for plan in (P.dense_int8_plan(*x, w[0].t(), w[1]), P.dequantize_plan(*x), P.quantize_plan(v.rows(40, 96))):
        first = lambda: plan.out if isinstance(plan.out, torch.Tensor) else plan.out[0]  # noqa: E731
        plan()
        want = first().clone()
        first().zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        plan(side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first(), want)


def test_types_and_devices_are_checked():
    v = Eight(40, torch.bfloat16)
    x, (q, s), (w, ws) = v.rows(6, 200), P.quantize(v.rows(6, 200)), P.quantize(v.rows(5, 200))
    dy, wt = v.rows(6, 5), v.weight(200, 5, "io")
    for call, match in (
            (lambda: P.quantize(q), "q has type|x has type"), (lambda: P.quantize(x, q=x.clone()), "q has type"),
            (lambda: P.quantize(x, scale=s.double()), "scale has type"), (lambda: P.dequantize(x, s), "q has type"),
            (lambda: P.dequantize(q, s, dtype=torch.int32), "out has type"), (lambda: P.dequantize(q, s.bfloat16()), "scale has type"),
            (lambda: P.dense_int8(x, s, w.t(), ws), "x has type"), (lambda: P.dense_int8(q, s, wt, ws), "weight has type"),
            (lambda: P.dense_int8(q, s, w.t(), ws, residual=dy, dtype=torch.float16), "residual has type"),
            (lambda: P.dense_int8(q, s, w.t(), ws, v.vector(5), out=torch.empty(6, 5, device="cuda:0")), "bias has type"),
            (lambda: P.dense_int8(q, s.cpu(), w.t(), ws), "must be a GPU tensor"),
            (lambda: P.dense_int8(q, s, w.t(), torch.ones(5, 2, device="cuda:0")[:, :1]), "must be contiguous"),
            (lambda: P.dense_backward_int8(dy, x, s, wt), "x has type"), (lambda: P.dense_backward_int8(dy, q, s, wt.float()), "weight has type"),
            (lambda: P.block_norm(x, x.float()), "residual has type"), (lambda: P.block_norm(x, x, gate=v.rows(3, 200, pad=1)), "contiguous"),
            (lambda: P.block_norm(x, x, weight=v.rows(1, 400)[0, ::2]), "contiguous"),
            (lambda: P.block_norm_backward(x, None, x, None, torch.ones(4, 6, device="cuda:0").half()), "stats has type")):
        with pytest.raises(ValueError, match=match):
            call()
    for call in (lambda: P.quantize_plan(x, q=torch.empty(6, 200, dtype=torch.int8, device="cuda:0").flip(0)[:, :0]),):
        with pytest.raises(ValueError, match="q has shape"):
            call()
