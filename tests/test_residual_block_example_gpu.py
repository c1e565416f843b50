"""The example stack of residual blocks: it runs, its gradients are those of its
formula at the checkpoints' values, and served rows are those of the operators one
after the other."""
import importlib.util
import os

import pytest
import torch

import block_oracle as B
import ff_oracle as O
import paper_2507_01040_amd as P

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_block_example",
                                                  os.path.join(ROOT, "examples", "residual_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_runs(example):
    stack, losses = example.train(steps=3, batch=256, channels=8)
    assert len(losses) == 3 and all(v == v for v in losses)
    for b in stack:
        assert all(bool(torch.isfinite(p.float()).all()) for p in b.params.values())


def test_gradients(example):
    # fp32, against the chain of formulas in 64 bits at the checkpoints' values; 1e-4 of the
    # largest gradient: sums of up to 300 terms and two norms (300^0.5 2^-24 each, some tens of
    # roundings) stay under 1e-5 of it
    block = example.Block(160, 300, dtype=torch.float32, seed=3)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    block.params = {k: v + 0.1 * torch.randn(v.shape, generator=gen, device="cuda:0") for k, v in block.params.items()}
    r, h = example.first_norm(example.clifford_rows(200, 40, (1, -1), 5, torch.float32))
    out, normed, saved = block.forward(r, h)
    dout, dnormed = (torch.randn(out.shape, generator=gen, device="cuda:0") for _ in range(2))
    dr, dh, grads = block.backward(dout, dnormed, saved)

    p = {k: v.cpu().double() for k, v in block.params.items()}
    (hq, hs), (preq, ps), (aq, as_), y, _, stats = saved
    h8, pre8, a8 = B.values(hq, hs), B.values(preq, ps), B.values(aq, as_)
    # each checkpoint within half a step of what it keeps
    for v, (q, s) in ((h, saved[0]),):
        step = s.cpu().double().repeat_interleave(128, 1)[:, :v.shape[1]]
        assert bool(((B.values(q, s) - v.cpu().double()).abs() <= 0.5001 * step).all())
    n = B.block_norm_backward(dout, dnormed, y, out, stats, block.params["gate"], 1.0, block.params["weight"], None,
                              block.params["next_weight"], True, True, torch.float32)
    dy = n["dx"][0]
    g = (dy @ p["w2"]) * O.slope(2, pre8)
    want = dict(w2=dy.t() @ a8, b2=dy.sum(0), w1=g.t() @ h8, b1=g.sum(0), gate=n["dgate"][0], weight=n["dweight"][0],
                next_weight=n["dnext_weight"][0])
    got = dict(grads, r=dr, h=dh)
    want.update(r=n["dresidual"][0], h=g @ p["w1"])
    for name, w in want.items():
        v = got[name].cpu().double()
        assert v.shape == w.shape, name
        assert float((v - w).abs().max()) <= 1e-4 * float(w.abs().max()), name


def test_serves(example):
    stack = [example.Block(256, 1024, seed=i) for i in range(2)]
    for rows in (1, 5, 200):
        r, h = example.first_norm(example.clifford_rows(rows, 64, (1, 1), 6, torch.bfloat16))
        serve = stack[0].server(r, h)
        for shift in (0.0, 0.25):  # new rows in the same buffers
            r.add_(shift)
            got = [t.clone() for t in serve()]
            p = stack[0].params
            (w1, s1), (w2, s2) = P.quantize(p["w1"]), P.quantize(p["w2"])
            a = P.dense_int8(*P.quantize(h), w1.t(), s1, p["b1"], act=P.ACT_GELU)
            y = P.dense_int8(*P.quantize(a), w2.t(), s2, p["b2"])
            want = P.block_norm(y, r, gate=p["gate"], weight=p["weight"], next_weight=p["next_weight"], rms=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            # and near the block in 64 bits without 8 bits: a step of a row's scale is 1 / 127 of
            # its largest value, 4 to 5 times a value's own size, so a rounding is off by 1 % of
            # the values, each product by 1.5 % of its rows (of both operands) and the norm's by 3 %
            d = {k: v.cpu().double() for k, v in p.items()}
            a = O.act(2, h.cpu().double() @ d["w1"].t() + d["b1"])
            y = a @ d["w2"].t() + d["b2"]
            n = y / (y.square().mean(1, keepdim=True) + 1e-5).sqrt() * d["weight"]
            out = r.cpu().double() + d["gate"] * n
            moved = (d["gate"] * n).norm()
            assert float((got[0].cpu().double() - out).norm()) <= 0.06 * float(moved) + 2.0 ** -8 * float(out.norm())
