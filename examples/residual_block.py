"""A stack of residual feed-forward blocks with a norm on either side, trained with
8-bit checkpoints and served with 8-bit products.

    python examples/residual_block.py

A batch of multivectors goes through a Clifford linear layer and becomes rows of
C * N_B features, r.  With h = n(r) the first block reads, every block is

    a = gelu(h w1 + b1),  y = a w2 + b2,
    r' = r + gate n(y),   h' = n(r')

with RMS norms n: block_norm takes both norms, the gate and the residual at once.
In training the forward pass keeps h, the pre-activations and a in 8 bits
(quantize), a scale for each 128 features, and the gradient reads them so
(dense_backward_int8).  Served, both products are those of 8-bit integers
(dense_int8), weights quantized once, rows as they come.  torch holds the memory,
the loss and the update.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2507_01040_amd as P  # noqa: E402


def _checkpoint(x):
    return P.quantize(x, group=P.residual_block.GROUP)


class Block:
    """One block's weights and its passes over (r, h)."""

    def __init__(self, features, hidden, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).to(dtype)
        ones = lambda: torch.ones(features, dtype=dtype, device=device)  # noqa: E731
        zeros = lambda n: torch.zeros(n, dtype=dtype, device=device)  # noqa: E731
        # the products' weights stored [out, in], as the 8-bit product reads them
        self.params = dict(w1=normal(hidden, features, scale=features ** -0.5), b1=zeros(hidden),
                           w2=normal(features, hidden, scale=hidden ** -0.5), b2=zeros(features),
                           gate=ones() * 0.5, weight=ones(), next_weight=ones())

    def _norms(self):
        p = self.params
        return dict(gate=p["gate"], weight=p["weight"], next_weight=p["next_weight"], rms=True)

    def forward(self, r, h):
        """(r', h') and what the gradient reads."""
        p = self.params
        a, pre = P.dense(h, p["w1"].t(), p["b1"], act=P.ACT_GELU, pre=True)
        y = P.dense(a, p["w2"].t(), p["b2"])
        out, normed, stats = P.block_norm(y, r, **self._norms())
        return out, normed, (_checkpoint(h), _checkpoint(pre), _checkpoint(a), y, out, stats)

    def backward(self, dout, dnormed, saved):
        """(dr, dh) of the block's inputs, and the parameters' gradients by name."""
        h, pre, a, y, out, stats = saved
        p = self.params
        n = P.block_norm_backward(dout, dnormed, y, out, stats, **self._norms())
        da, dw2, db2 = P.dense_backward_int8(n.dx, *a, p["w2"].t())
        dh, dw1, db1 = P.dense_backward_int8(da, *h, p["w1"].t(), pre=pre[0], pre_scale=pre[1], act=P.ACT_GELU)
        return n.dresidual, dh, dict(w1=dw1.t(), b1=db1, w2=dw2.t(), b2=db2, gate=n.dgate, weight=n.dweight,
                                     next_weight=n.dnext_weight)

    def server(self, r, h):
        """A call that takes what the buffers r and h hold through the block, and returns
        (r', h'): weights in 8 bits, every buffer and check once."""
        p = self.params
        w1, s1 = P.quantize(p["w1"])
        w2, s2 = P.quantize(p["w2"])
        rows = P.quantize_plan(h)
        first = P.dense_int8_plan(*rows.out, w1.t(), s1, p["b1"], act=P.ACT_GELU)
        hidden = P.quantize_plan(first.out)
        second = P.dense_int8_plan(*hidden.out, w2.t(), s2, p["b2"])
        norms = P.block_norm_plan(second.out, r, **self._norms())

        def serve():
            for plan in (rows, first, hidden, second, norms):
                plan()
            return norms.out[:2]
        return serve


def clifford_rows(batch, channels, g, seed, dtype):
    """Rows of a Clifford linear layer's output, one for each multivector."""
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    blades = 1 << len(g)
    x = torch.randn((batch, channels, blades), generator=gen, device="cuda:0")
    w = torch.randn((channels, channels, blades), generator=gen, device="cuda:0") * (channels * blades) ** -0.5
    return P.linear(x, w, torch.zeros(channels, blades, device="cuda:0"), g).flatten(1).to(dtype)


def first_norm(r):
    """(r, h) of the first block: the norm before it, of the rows as they are."""
    zero = torch.zeros_like(r)
    return P.block_norm(zero, r, after=False, rms=True)[:2]


def train(steps=100, batch=4096, channels=32, blocks=2, rate=0.02, dtype=torch.bfloat16, log=lambda s: None):
    """Trains a stack to reproduce a fixed map of its rows; (stack, losses)."""
    features = 4 * channels
    stack = [Block(features, 4 * features, dtype, seed=i) for i in range(blocks)]
    r = clifford_rows(batch, channels, (1, 1), 7, dtype)
    gen = torch.Generator(device="cuda:0").manual_seed(8)
    turn = torch.randn((features, features), generator=gen, device="cuda:0") * features ** -0.5
    target = r.float() + torch.tanh(r.float() @ turn)
    losses = []
    for step in range(steps):
        out, h = first_norm(r)
        saved = []
        for b in stack:
            out, h, s = b.forward(out, h)
            saved.append(s)
        off = out.float() - target
        losses.append(float(off.square().mean()))
        log("step %d: loss %.4f" % (step, losses[-1]))
        # only r' of the last block has a loss: its h' has none
        dout, dh = (off * (2.0 / off.shape[0])).to(dtype), torch.zeros_like(out)
        for b, s in zip(reversed(stack), reversed(saved)):
            dout, dh, grads = b.backward(dout, dh, s)
            for name, g in grads.items():
                p = b.params[name]
                p.copy_(p.float() - rate * g.float())
    return stack, losses


if __name__ == "__main__":
    stack, losses = train(log=lambda s: print(s) if s.split(":")[0].endswith("0") else None)
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    r, h = first_norm(clifford_rows(4, 32, (1, 1), 9, torch.bfloat16))
    for b in stack:
        r, h = b.server(r, h)()
    torch.cuda.synchronize()
    print("served rows:", tuple(r.shape), "finite:", bool(torch.isfinite(r.float()).all()))
