"""Whose memory the Clifford layers' calls write, without a GPU: CPU tensors
stand for those on the GPU and the library's entry points do nothing."""
import pytest
import torch

import paper_2507_01040_amd as P
from test_feed_forward_arguments import _Stream, library, streams  # noqa: F401


@pytest.fixture
def clifford(library, monkeypatch):  # noqa: F811
    monkeypatch.setattr(P, "_check_dev", lambda *a, **kw: None)


_inputs = {}  # of the calls


def _calls(stream):
    x, f = torch.zeros(2, 3, 8, 8, 4), torch.zeros(3, 3, 3, 3, 4)
    v, w = torch.zeros(2, 3, 4), torch.zeros(3, 5, 4)
    b, g = torch.zeros(3, 4), (1, 1)
    layer, act = (f, b, None), (P.AGG_LINEAR, (0, 1), torch.zeros(5, 2), torch.zeros(5))
    _inputs.update(conv_nd=(x, f, b), conv_plan=(x, f, b), linear=(v, w, act[2], act[3]), act_nd=(x,), block2=(x, f, b),
                   block2_plan=(x, f, b))
    return {"conv_nd": lambda: P.conv_nd(x, f, b, g, stream=stream),
            "conv_plan": lambda: P.conv_plan(x, f, b, g, stream=stream),
            "linear": lambda: P.linear(v, w, None, g, act=act, stream=stream),
            "act_nd": lambda: P.act_nd(x, P.AGG_SUM, (0, 1), stream=stream),
            "block2": lambda: P.block2(x, layer, layer, g, stream=stream),
            "block2_plan": lambda: P.block2_plan(x, layer, layer, g, stream=stream)}


@pytest.mark.parametrize("op", _calls(None))
def test_buffers_are_the_streams_own(clifford, streams, op):  # noqa: F811
    for stream, name in ((None, "first"), (_Stream(), "handle 1234")):
        call = _calls(stream)[op]
        streams["made"].clear()
        streams["recorded"].clear()
        got = call()
        inputs = set(_inputs[op])
        assert len(streams["made"]) == (2 if op.startswith("block2") else 1)
        assert {s for _, s in streams["made"]} == {name} and streams["current"] == "first"
        used = {p for p, _ in streams["made"]} | {t.data_ptr() for t in inputs}
        assert set(streams["recorded"]) == (set() if stream is None else {(p, "first") for p, _ in streams["made"]} |
                                            {(p, name) for p in used})
        if op.endswith("_plan"):
            streams["recorded"].clear()
            got(7)
            assert set(streams["recorded"]) == {(p, "handle 7") for p in used}


@pytest.mark.gpu
def test_calls_on_another_stream():
    # memory that the current stream has just freed is not what they write, and
    # the results are the same
    gen = torch.Generator(device="cuda:0").manual_seed(3)

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda:0")
    x, f, v, w = rand(4, 8, 20, 20, 4), rand(8, 8, 3, 3, 4), rand(64, 16, 4), rand(16, 16, 4)
    g, layer = (1, -1), (f, None, None)
    side = torch.cuda.Stream()
    for call in (lambda s: P.conv_nd(x, f, None, g, stream=s), lambda s: P.linear(v, w, None, g, stream=s),
                 lambda s: P.act_nd(x, P.AGG_SUM, (0, 1), stream=s), lambda s: P.block2(x, layer, layer, g, stream=s)):
        want = call(None)
        torch.cuda.synchronize()
        freed = [torch.empty_like(want) for _ in range(4)]
        places = {t.data_ptr() for t in freed}
        del freed
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        assert got.data_ptr() not in places
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)


def test_current_device(monkeypatch):
    # without a stream the call goes to the current device's: tensors of another one
    # are refused
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream())
    assert P._stream_ptr(None, torch.device("cuda:0")) == 0x1234
    assert P._stream_ptr(_Stream(), torch.device("cuda:1")) == 0x1234
    with pytest.raises(ValueError, match="the tensors are on cuda:1, but the current device is cuda:0"):
        P._stream_ptr(None, torch.device("cuda:1"))


@pytest.mark.gpu
def test_inputs_freed_after_a_call_on_another_stream():
    # a temporary among the arguments is not given to others while the other stream
    # still has it to read
    w, f = torch.randn(256, 256, device="cuda:0"), torch.randn(8, 8, 3, 3, 4, device="cuda:0")
    side = torch.cuda.Stream()
    for make, call in ((lambda: torch.ones(512, 256, device="cuda:0"), lambda x: P.dense(x, w, stream=side)),
                       (lambda: torch.ones(4, 8, 20, 20, 4, device="cuda:0"),
                        lambda x: P.conv_nd(x, f, None, (1, 1), stream=side))):
        x = make()
        want = call(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)  # about a tenth of a second
        side.wait_stream(torch.cuda.current_stream())
        place = x.data_ptr()
        got = call(x)
        del x
        others = [make().fill_(float("nan")) for _ in range(4)]
        assert place not in {t.data_ptr() for t in others}
        torch.cuda.synchronize()
        assert torch.equal(got, want)
