"""The 8-bit operators and the block norm on the GPU where their kernels' loops run long
and their choices meet: the steady loop of the weight's gradient from 8 bits, exactly the
roundings that the gradient names, parts of several passes, every number of gates with
every norm, in place too, and scales of both signs."""
import itertools

import pytest
import torch

import block_oracle as B
import ff_oracle as O
import paper_2507_01040_amd as P
from block_cases import STEADY
from test_feed_forward_gpu import DTYPES, KEY, STEP, Draw, ids, rng
from test_residual_block_gpu import EPS, Eight, _check_gradient, _check_norm, _gradient, _norm_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("size", [s for s, _ in STEADY], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_steady_loop_of_the_weight_gradient(dtype, size, order):
    (M, K, N), i = size, [s for s, _ in STEADY].index(size)
    v = Eight(50 + i, dtype)
    xg, pg = (-(-K // 128) if i % 2 else 1), (-(-N // 128) if i < 2 else 1)
    x, xs, w = v.int8(M, K, pad=3 * (i // 2)), v.scale(M, xg, 0.01), v.weight(K, N, order)
    pre, ps, dy = v.int8(M, N), v.scale(M, pg, 0.01), v.rows(M, N, pad=i % 2)
    a = (P.ACT_GELU, P.ACT_SILU)[(i + (order == "oi")) % 2]
    drop = (0.2, rng()) if i % 2 else None
    got = P.dense_backward_int8(dy, x, xs, w, pre, ps, act=a, dropout=drop)
    for g, ref, name in zip(got, B.dense_backward_int8(dy, x, xs, w, pre, ps, a, drop and (0.2, (KEY, STEP)), dtype), ("dx", "dw", "dbias")):
        O.check(g, ref, name)
    again = P.dense_backward_int8(dy, x, xs, w, pre, ps, act=a, dropout=drop)
    assert all(torch.equal(g, h) for g, h in zip(got, again))


@pytest.mark.parametrize("act", [P.ACT_GELU, P.ACT_SILU])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=ids)
def test_gradient_has_the_roundings_that_it_names_and_no_others(dtype, grouped, act):
    # Against sums in 64 bits of the operands as the header has them rounded (bf16: g for dx,
    # scale g for dw; fp16: none but two bf16 parts for dw), rounded to the type.  u = half a
    # step at 1.  A step is u to 2 u of a value.  Operands: f' is within COST U, so at most
    # 2 COST U / u = 2^-11 of the operands round to the other neighbour, 2 u away: 0.044 u in
    # the 2-norm (fp16's two parts: 2^-17 = 2^-6 u).  fp32 sums of n independent terms, whose
    # partial sums are no larger than the result: LAMBDA n^0.5 U = 2.4e-5, 0.006 u (fp16: 0.05 u).
    # Together e <= 0.07 u before the output's rounding, which then differs in e / step of the
    # values by a step: (e 2 u)^0.5 <= 0.38 u.  A rounding more is 0.6 u and more.
    M, K, N, p = 2600, 512, 640, 0.1
    u = O.UNIT[dtype]
    v = Eight(60, dtype)
    group = 128 if grouped else None
    (q, s), (pre, ps), w = P.quantize(v.rows(M, K), group=group), P.quantize(v.rows(M, N), group=group), v.weight(K, N, "io")
    dy = v.rows(M, N, scale=0.05)
    dx, dw, _ = P.dense_backward_int8(dy, q, s, w, pre, ps, act=act, dropout=(p, rng()))
    g = dy.cpu().double() * O.slope(act, B.values(pre, ps)) * (O.mask((p, (KEY, STEP)), M, N) * (1 - p))

    def off(got, want):
        want = want.to(dtype).double()
        return float((got.cpu().double() - want).norm() / want.norm()) / u
    if dtype == torch.bfloat16:
        assert off(dx, (g.bfloat16().double() @ w.cpu().double().t()) / (1 - p)) <= 0.38
    want = []
    for c in range(0, K, 128):
        each = g * s[:, c // 128 if grouped else 0].cpu().double()[:, None]
        want.append(q[:, c:c + 128].cpu().double().t() @ (each.bfloat16().double() if dtype == torch.bfloat16 else each) / (1 - p))
    assert off(dw, torch.cat(want)) <= 0.38


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_int8_scales_of_both_signs(dtype):
    # scales far from one whose product is an ordinary float, of either sign: few rows, tiles,
    # a split contraction, panels
    for M, K, N in ((3, 20000, 40), (70, 20016, 72), (300, 130, 65), (2100, 112, 1030)):
        v = Eight(61, dtype)
        x, w = torch.full((M, K), 127, dtype=torch.int8, device="cuda:0"), torch.full((N, K), -127, dtype=torch.int8, device="cuda:0")
        w[::3] = v.int8(w[::3].shape[0], K)
        xs, ws = v.scale(M), v.scale(N, size=1 / (16000 * K))
        xs[1::2] *= -1
        ws[::4] *= -1
        for far in (118, -118):
            a, b = torch.ldexp(xs, torch.tensor(far)), torch.ldexp(ws, torch.tensor(-far))
            y = P.dense_int8(x, a, w.t(), b, dtype=dtype)
            O.check(y, B.dense_int8(x, a, w.t(), b, None, 0, None, dtype), "y of %s" % ((M, K, N, far),))


CHOICES = list(itertools.product(((True, True), (True, False), (False, True)), (False, True)))


def _chosen(dtype, size, gates, norms, rms, seed):
    after, before = norms
    gate = None if gates == 0 else Draw(seed, dtype).vector(size[1]) if gates == 1 else Draw(seed, dtype).rows(gates, size[1])
    c = _norm_case(dtype, size, 0, after=after, before=before, rms=rms, gate=gate, scale=(0.5, -2.0)[seed % 2])
    if not after:
        c["weight"] = c["bias"] = None
    if not before:
        c["next_weight"] = c["next_bias"] = None
    return c


@pytest.mark.parametrize("size,gates", [((120, 96), (0, 1, 4, 20, 60, 120)), ((64, 300), (0, 2, 32, 64)), ((96, 777), (1, 4, 48)),
                                        ((60, 2049), (1, 20, 30)), ((36, 5000), (0, 3, 18)), ((24, 8200), (0, 1, 2, 12, 24))], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_of_every_choice(dtype, size, gates):
    for n, (norms, rms) in enumerate(CHOICES):
        for i in gates:
            c = _chosen(dtype, size, i, norms, rms, 70 + n)
            got = P.block_norm(**c, eps=EPS)
            _check_norm(c, got, dtype)
            k = _gradient(c, size, dtype, n + i)
            grads = P.block_norm_backward(**k)
            _check_gradient(k, grads, dtype)
            # in place: the same bits
            for to in (("residual", "x"), ("x", "residual")):
                at = dict(c, x=c["x"].clone(), residual=c["residual"].clone())
                into = dict(out=at[to[0]], normed=at[to[1]] if norms[1] else None)
                for a, b in zip(P.block_norm(**at, eps=EPS, **into)[:-1], got[:-1]):
                    assert torch.equal(a, b)
            if k["dout"] is not None and k["dnormed"] is not None:
                for to in (("dout", "dnormed"), ("dnormed", "dout")):
                    at = dict(k, dout=k["dout"].clone(), dnormed=k["dnormed"].clone())
                    for a, b in zip(P.block_norm_backward(**at, dx=at[to[0]], dresidual=at[to[1]]), grads):
                        assert a is b is None or torch.equal(a, b)


@pytest.mark.parametrize("gates", [20, 64, 640, 1280])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_block_norm_gradient_of_many_gates(dtype, gates):
    for n, (norms, rms) in enumerate(CHOICES):
        c = _chosen(dtype, (1280, 260), gates, norms, rms, 80 + n)
        k = _gradient(c, (1280, 260), dtype, 1)
        _check_gradient(k, P.block_norm_backward(**k), dtype)


@pytest.mark.parametrize("size", [(70000, 128), (20000, 300), (9000, 1000)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=ids)
def test_block_norm_gradient_of_parts_in_several_passes(dtype, size):
    for i, gates in enumerate((1, 50)):
        c = _chosen(dtype, size, gates, (True, True), i == 1, 90 + i)
        k = _gradient(c, size, dtype, 1)
        _check_gradient(k, P.block_norm_backward(**k), dtype)
