"""A residual feed-forward block between Clifford linear layers, trained and
served through the library's operators.

    python examples/feed_forward.py

A batch of multivectors goes through a Clifford linear layer (as in a network
of them) and becomes rows of C * N_B features.  The block on top of it,

    h = layer_norm(x);  a = dropout(gelu(h w1 + b1));  y = x + dropout(a w2 + b2),

is trained to reproduce a fixed map of its rows: every product, norm,
activation, dropout and gradient runs in the library's kernels; torch holds the
memory, the loss and the update.  Then single rows are served through plans.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2507_01040_amd as P  # noqa: E402


class FeedForward:
    """The block's weights (in the library's order, [features in, features
    out]) and its passes."""

    def __init__(self, features, hidden, p=0.1, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).to(dtype)
        self.p = p
        # the generator's key and step: every forward pass of training takes a new step
        self.rng1 = torch.tensor([seed, 0], dtype=torch.int64, device=device)
        self.rng2 = torch.tensor([seed + 1, 0], dtype=torch.int64, device=device)
        self.params = [torch.ones(features, dtype=dtype, device=device),
                       torch.zeros(features, dtype=dtype, device=device),
                       normal(features, hidden, scale=features ** -0.5),
                       torch.zeros(hidden, dtype=dtype, device=device),
                       normal(hidden, features, scale=0.1 * hidden ** -0.5),
                       torch.zeros(features, dtype=dtype, device=device)]

    def train_forward(self, x):
        nw, nb, w1, b1, w2, b2 = self.params
        self.rng1[1] += 1
        self.rng2[1] += 1
        h, mean, rstd = P.layer_norm(x, nw, nb)
        a, pre = P.dense(h, w1, b1, act=P.ACT_GELU, dropout=(self.p, self.rng1), pre=True)
        y = P.dense(a, w2, b2, dropout=(self.p, self.rng2), residual=x)
        return y, (x, h, mean, rstd, a, pre)

    def backward(self, dy, saved):
        """The gradients of x and of the parameters; the masks are formed again."""
        x, h, mean, rstd, a, pre = saved
        nw, _, w1, _, w2, _ = self.params
        da, dw2, db2 = P.dense_backward(dy, a, w2, dropout=(self.p, self.rng2))
        dh, dw1, db1 = P.dense_backward(da, h, w1, pre=pre, act=P.ACT_GELU, dropout=(self.p, self.rng1))
        dx, dnw, dnb = P.layer_norm_backward(dh, x, mean, rstd, nw, dresidual=dy)
        return dx, [dnw, dnb, dw1, db1, dw2, db2]

    def server(self, x):
        """The block without dropout for rows of x's shape, as plans on fixed
        buffers: call it after writing new rows to x."""
        nw, nb, w1, b1, w2, b2 = self.params
        norm = P.layer_norm_plan(x, nw, nb)
        first = P.dense_plan(norm.out[0], w1, b1, act=P.ACT_GELU)
        second = P.dense_plan(first.out, w2, b2, residual=x)

        def serve():
            norm()
            first()
            return second()
        return serve


def clifford_rows(batch, channels, g, seed, dtype, device="cuda:0"):
    """Rows of channels * N_B features from a Clifford linear layer."""
    nb = 1 << len(g)
    gen = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn((batch, channels, nb), generator=gen, device=device)
    w = torch.randn((channels, channels, nb), generator=gen, device=device) * (channels * nb) ** -0.5
    return P.linear(x, w, None, g).flatten(1).to(dtype)


def train(steps=60, batch=4096, channels=32, g=(1, 1), rate=0.015, dtype=torch.bfloat16):
    """Trains the block; returns it and the losses."""
    features = channels * (1 << len(g))
    block = FeedForward(features, 4 * features, dtype=dtype)
    masters = [p.float() for p in block.params]
    target = torch.randn((features, features), generator=torch.Generator(device="cuda:0").manual_seed(9),
                         device="cuda:0") * (0.5 * features ** -0.5)
    losses = []
    for step in range(steps):
        x = clifford_rows(batch, channels, g, 100 + step, dtype)
        want = x.float() + torch.tanh(x.float() @ target)
        y, saved = block.train_forward(x)
        off = y.float() - want
        losses.append(float(off.square().mean()))
        _, grads = block.backward((off * (2.0 / batch)).to(dtype), saved)
        for master, param, grad in zip(masters, block.params, grads):
            master.sub_(grad.float(), alpha=rate)
            param.copy_(master)
    return block, losses


def main():
    block, losses = train()
    print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], len(losses)))
    row = clifford_rows(1, 32, (1, 1), 7, torch.bfloat16)
    serve = block.server(row)
    for _ in range(10):
        serve()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(200):
        serve()
    end.record()
    torch.cuda.synchronize()
    print("one row of %d features: %.1f us" % (row.shape[1], start.elapsed_time(end) * 5))


if __name__ == "__main__":
    main()
