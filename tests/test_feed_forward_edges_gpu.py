"""Edges of the feed-forward operators on the GPU, against the plain
implementations in 64 bits of ff_oracle.py (which derives the bounds)."""
import pytest
import torch

import ff_oracle as O
import paper_2507_01040_amd as P
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
