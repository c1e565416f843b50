"""What the feed-forward binding passes to the library, without a GPU: the
calls' arguments are taken where the library would be called, and CPU tensors
stand for those on the GPU."""
import pytest
import torch

import paper_2507_01040_amd as P
from paper_2507_01040_amd import feed_forward as F

DENSE_BACKWARD = ("dtype M K N dy lddy x ldx w ldw order pre ldp act drop dx lddx dw lddw dbias ws "
                  "ws_bytes stream").split()


class _Library:
    """Entry points that record their arguments; workspaces of 256 bytes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 256

        def entry(*args):
            self.calls.append((name, args))
            return P.CLIFF_OK
        entry.argtypes = [lambda v: v] * 40
        return entry


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(P, "load", lambda *a: lib)
    monkeypatch.setattr(P, "_stream_ptr", lambda stream, device: 0)
    monkeypatch.setattr(F, "_check_dev", lambda *a, **kw: None)
    return lib


def _stored(order, ld, K, N):
    """A weight [K, N] of the order with that row stride, inside a larger buffer."""
    if order:
        return torch.zeros(N + 1, ld)[:N, :K].t()
    return torch.zeros(K + 1, ld)[:K, :N]


def _written(args, K, N):
    """Byte offset from dw of every element (k, n) as the header lays them out."""
    k, n = torch.arange(K)[:, None], torch.arange(N)[None, :]
    return (n * args["lddw"] + k if args["order"] else k * args["lddw"] + n) * 4


def _meant(t):
    K, N = t.shape
    return (torch.arange(K)[:, None] * t.stride(0) + torch.arange(N)[None, :] * t.stride(1)) * 4


@pytest.mark.parametrize("given", [None, "io", "oi", "wide"])
@pytest.mark.parametrize("order", ["io", "oi"])
@pytest.mark.parametrize("K,N,pad", [(1, 512, 6), (1, 512, 0), (512, 1, 6), (512, 1, 0), (1, 1, 3), (1, 2, 0), (2, 1, 5),
                                     (7, 5, 0), (7, 5, 2)], ids=str)
def test_weight_gradient_goes_where_its_tensor_is(library, K, N, pad, order, given):
    # one input or output feature: the strides of [K, N] and of a stored [N, K] do
    # not tell the order
    w = _stored(order == "oi", (K if order == "oi" else N) + pad, K, N)
    dweight = None
    if given == "wide":
        dweight = _stored(order == "oi", (K if order == "oi" else N) + 9, K, N)
    elif given:
        dweight = _stored(given == "oi", K if given == "oi" else N, K, N)
    x, dy = torch.zeros(3, K), torch.zeros(3, N)
    try:
        out = P.dense_backward(dy, x, w, dweight=dweight)[1]
    except ValueError as e:
        # refused: only a gradient that the weight's order cannot hold
        assert "order of the weight" in str(e) and given in ("io", "oi") and min(K, N) > 0
        got_order = F._weight_order(w)[0]
        sk, sn = dweight.stride()
        assert (sk != 1 and K > 1 or sn < K and N > 1) if got_order else (sn != 1 and N > 1 or sk < N and K > 1)
        return
    name, args = library.calls[-1]
    assert name == "cliffconv_dense_backward"
    args = dict(zip(DENSE_BACKWARD, args))
    assert args["dw"] == out.data_ptr() and out.shape == (K, N)
    if dweight is not None:
        assert out is dweight
    assert torch.equal(_written(args, K, N), _meant(out))
    # and inside its storage
    last = out.storage_offset() * 4 + int(_written(args, K, N).max()) + 4
    assert last <= out.untyped_storage().nbytes()
    # the weight is read where it is, in the same order
    k, n = torch.arange(K)[:, None], torch.arange(N)[None, :]
    read = (n * args["ldw"] + k if args["order"] else k * args["ldw"] + n) * 4
    assert torch.equal(read, _meant(w))
    least = K if args["order"] else N
    assert args["ldw"] >= least and args["lddw"] >= least


class _Stream:
    cuda_stream = 0x1234


@pytest.fixture
def streams(monkeypatch):
    """Streams by name: which one is current, where tensors were allocated and
    which ones they were recorded on."""
    log = dict(current="first", made=[], recorded=[])

    class Use:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            self.before, log["current"] = log["current"], self.s

        def __exit__(self, *a):
            log["current"] = self.before
    empty = torch.empty

    def noted(*a, **kw):
        t = empty(*a, **kw)
        log["made"].append((t.data_ptr(), log["current"]))
        return t
    monkeypatch.setattr(torch.cuda, "stream", Use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: log["current"])
    monkeypatch.setattr(P, "_torch_stream", lambda s, d: "handle %x" % (s if isinstance(s, int) else s.cuda_stream))
    monkeypatch.setattr(torch, "empty", noted)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log["recorded"].append((t.data_ptr(), s)))
    return log


def _calls(stream):
    """(call, its inputs) of every operator."""
    x, w, r = torch.zeros(6, 8), torch.zeros(8, 5), torch.zeros(2, dtype=torch.int64)
    dy, v, b = torch.zeros(6, 5), torch.zeros(6), torch.zeros(5)
    return {"dense": (lambda: P.dense_plan(x, w, b, dropout=(0.5, r), residual=dy, pre=True, stream=stream),
                      (x, w, b, r, dy)),
            "dense_backward": (lambda: P.dense_backward_plan(dy, x, w, dropout=(0.5, r), stream=stream), (dy, x, w, r)),
            "layer_norm": (lambda: P.layer_norm_plan(x, stream=stream), (x,)),
            "layer_norm_backward": (lambda: P.layer_norm_backward_plan(x, x, v, v, stream=stream), (x, v)),
            "dropout": (lambda: P.dropout_plan(x, 0.5, r, stream=stream), (x, r))}


@pytest.mark.parametrize("op", _calls(None))
def test_buffers_are_the_streams_own(library, streams, op):
    # memory that the current stream has freed may still be read there: what a
    # call on another stream writes is allocated for that one; what it reads may be
    # freed after the call, and is noted as used there
    for stream, name in ((None, "first"), (_Stream(), "handle 1234")):
        call, inputs = _calls(stream)[op]
        streams["made"].clear()
        streams["recorded"].clear()
        plan = call()
        assert streams["made"] and {s for _, s in streams["made"]} == {name}
        assert streams["current"] == "first"
        # and the caller, who reads it on the current stream, may free it at any time
        used = {p for p, _ in streams["made"]} | {t.data_ptr() for t in inputs}
        assert set(streams["recorded"]) == (set() if stream is None else {(p, "first") for p, _ in streams["made"]} |
                                            {(p, name) for p in used})
        # a plan's call on a third stream, as torch's or by its handle
        for third in (7, type("S", (), {"cuda_stream": 8})()):
            streams["recorded"].clear()
            plan(third)
            third = "handle %x" % getattr(third, "cuda_stream", third)
            assert set(streams["recorded"]) == {(p, third) for p in used}


@pytest.mark.parametrize("op", ["dense", "dense_backward", "layer_norm", "layer_norm_backward", "dropout"])
def test_tensors_that_require_a_gradient(library, monkeypatch, op):
    # autograd would not see the call: refused while it records, for each tensor
    monkeypatch.setattr(F, "_check_dev", lambda t, name, *a, **kw: F._check_grad(t, name))

    def tensors():
        x, w, r = torch.zeros(6, 8), torch.zeros(8, 5), torch.zeros(2, dtype=torch.int64)
        dy, v, m = torch.zeros(6, 5), torch.zeros(8), torch.zeros(6)
        return {"dense": dict(x=x, weight=w, bias=torch.zeros(5), residual=dy, out=torch.zeros(6, 5)),
                "dense_backward": dict(dy=dy, x=x, weight=w, dx=torch.zeros(6, 8), dweight=torch.zeros(8, 5),
                                       dbias=torch.zeros(5)),
                "layer_norm": dict(x=x, weight=v, bias=torch.zeros(8), out=torch.zeros(6, 8)),
                "layer_norm_backward": dict(dy=x, x=torch.zeros(6, 8), mean=m, rstd=torch.zeros(6), weight=v,
                                            dresidual=torch.zeros(6, 8)),
                "dropout": dict(x=x, p=0.5, rng=r, residual=torch.zeros(6, 8))}[op]
    call = getattr(P, op)
    call(**tensors())
    for name, t in tensors().items():
        if not isinstance(t, torch.Tensor) or t.dtype != torch.float32:
            continue
        kw = tensors()
        kw[name].requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            call(**kw)
        with torch.no_grad():
            call(**kw)
        with torch.inference_mode():
            call(**kw)
        kw[name] = kw[name].detach()
        call(**kw)
