"""The example block: it learns, its gradients are those of its formula, and
the served rows are those of the forward pass without dropout."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward_example",
                                                  os.path.join(ROOT, "examples", "feed_forward.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain(block, x, masks=None):
    # the block in float64 from its formula; masks: scaled dropout masks
    nw, nb, w1, b1, w2, b2 = block
    m1, m2 = masks if masks else (1.0, 1.0)
    c = x - x.mean(1, keepdim=True)
    h = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * nw + nb
    a = h @ w1 + b1
    a = a * 0.5 * torch.special.erfc(-a * 0.5 ** 0.5) * m1
    return x + (a @ w2 + b2) * m2


def test_learns(example):
    _, losses = example.train(steps=60, batch=1024)
    assert losses[-1] < 0.5 * losses[0], (losses[0], losses[-1])


def test_gradients_against_autograd(example):
    # fp32 block against float64 autograd with the same masks; 1e-4 of the largest
    # gradient: three layers of fp32 sums of up to 256 terms (256^0.5 2^-24 each, some
    # tens of roundings) stay under 1e-5 of it
    import ff_oracle as O
    block = example.FeedForward(48, 80, p=0.25, dtype=torch.float32, seed=3)
    x = example.clifford_rows(256, 12, (1, -1), 5, torch.float32)
    y, saved = block.train_forward(x)
    dy = torch.randn(y.shape, generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0")
    dx, grads = block.backward(dy, saved)
    masks = [O.mask((0.25, tuple(r.tolist())), 256, d) for r, d in ((block.rng1, 80), (block.rng2, 48))]
    leaves = [p.cpu().double().requires_grad_() for p in block.params]
    xd = x.cpu().double().requires_grad_()
    out = _plain(leaves, xd, masks)
    assert float((out.detach() - y.cpu().double()).abs().max()) < 1e-4
    out.backward(dy.cpu().double())
    for got, leaf in zip([dx, *grads], [xd, *leaves]):
        assert float((got.cpu().double() - leaf.grad).abs().max()) <= 1e-4 * float(leaf.grad.abs().max())


def test_serves(example):
    block = example.FeedForward(64, 256, dtype=torch.float32, seed=4)
    for rows in (1, 3, 100):
        x = example.clifford_rows(rows, 16, (1, 1), 6, torch.float32)
        serve = block.server(x)
        for shift in (0.0, 0.5):  # new rows in the same buffer
            x.add_(shift)
            want = _plain([p.cpu().double() for p in block.params], x.cpu().double())
            assert float((serve().cpu().double() - want).abs().max()) < 1e-4
