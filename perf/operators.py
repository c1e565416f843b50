"""The operators of a pre-norm residual feed-forward block that are measured:
dense layers (matrix product with bias, activation, dropout and residual in
its epilogue) and their gradients, layer norm forward and backward, and dropout
from a counter-based generator.

Rows are tokens, or the flattened multivectors (C * N_B features) between two
Clifford linear layers.  Sizes are those of the repository's linear layers
(32 channels of 4 blades: 128 features, up to 2^20 rows) and generic ones of
feed-forward parts; `draw` spreads over the same ranges: one row to many, odd
widths, padded rows, every type, activation and weight order.

The plain forms compute in float32 and round once.  `exact` computes in
float64 and has its own generator.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")  # in the order of the library's constants
EPS = 1e-5


def _dense(name, t, M, K, N, act, bias=True, p=0.0, residual=False, pre=False, order="io", pad=0):
    # order: the weight is [in, out] ("io") or a transposed view of [out, in] ("oi");
    # pad: elements between the rows of x beyond its width
    c = {"op": "dense", "type": t, "M": M, "K": K, "N": N, "act": act, "bias": bias, "p": p,
         "residual": residual, "pre": pre, "order": order, "pad": pad}
    return dict(c, name=name) if name else c


def _grad(name, t, M, K, N, act, bias=True, p=0.0, order="io", pad=0):
    c = {"op": "dense_backward", "type": t, "M": M, "K": K, "N": N, "act": act, "bias": bias,
         "p": p, "order": order, "pad": pad}
    return dict(c, name=name) if name else c


def _norm(name, t, rows, d, pad=0):
    c = {"op": "layer_norm", "type": t, "rows": rows, "d": d, "pad": pad}
    return dict(c, name=name) if name else c


def _norm_grad(name, t, rows, d, residual=False, pad=0):
    c = {"op": "layer_norm_backward", "type": t, "rows": rows, "d": d, "residual": residual,
         "pad": pad}
    return dict(c, name=name) if name else c


def _drop(name, t, rows, d, p, residual=False, pad=0):
    c = {"op": "dropout", "type": t, "rows": rows, "d": d, "p": p, "residual": residual, "pad": pad}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through a block's first layer while serving: latency and the weight's read
        _dense("dense_one_row", "bf16", 1, 1024, 4096, "silu"),
        # a small batch of tokens while serving, the second layer with its residual, a weight
        # stored [out, in]
        _dense("dense_few_rows", "fp16", 24, 4096, 4096, "none", residual=True, order="oi"),
        # a ragged batch: no size a multiple of a vector, rows of x padded
        _dense("dense_odd", "fp16", 1003, 777, 1531, "gelu", p=0.1, residual=True, pad=5),
        # the framework's own rows: 32 channels of 4 blades, widened four times
        _dense("dense_multivectors", "fp32", 1 << 17, 128, 512, "gelu"),
        # the training pass of a large first layer, pre-activation kept for the gradient
        _dense("dense_large", "bf16", 4096, 4096, 8192, "gelu", p=0.1, pre=True),
        # the gradient of an ordinary feed-forward layer in training
        _grad("dense_grad", "bf16", 8192, 2048, 2048, "gelu", p=0.1),
        # the gradient of the framework's rows: a long sum over rows, few weights
        _grad("dense_grad_multivectors", "fp32", 1 << 16, 128, 512, "silu"),
        # the norm of a few tokens while serving: latency
        _norm("norm_few_rows", "bf16", 4, 4096),
        # the norm between two of the framework's linear layers, at their largest batch
        _norm("norm_multivectors", "fp32", 1 << 20, 128),
        # the norm's gradient in training, with the residual branch's gradient added
        _norm_grad("norm_grad", "bf16", 16384, 4096, residual=True),
        # dropout on a block's output in training
        _drop("dropout_large", "bf16", 16384, 4096, 0.1, residual=True),
        # dropout on a small ragged batch, padded rows
        _drop("dropout_odd", "fp32", 1001, 777, 0.25, pad=3),
    ]


def _size(n):
    # 3072 stays out of the cases
    return n + 1 if n == 3072 else n


def _log(rng, lo, hi):
    return _size(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    # an odd width half of the time, else a power of two or 5/4 of one
    w = _log(rng, lo, hi)
    if rng.random() < 0.5:
        return _size(w | 1)
    w = 1 << (w.bit_length() - 1)
    return _size(min(hi, w * rng.choice((4, 4, 5)) // 4))


def draw(rng):
    t = rng.choice(("fp32", "bf16", "fp16"))
    pad = rng.choice((0, 0, rng.randint(1, 16), 64))
    p = rng.choice((0.0, 0.1, round(rng.uniform(0.05, 0.6), 3)))
    op = rng.choice(("dense", "dense", "dense_backward", "dense_backward", "norm", "norm_grad", "drop"))
    if op.startswith("dense"):
        most = 4096 * 4096 * 8192 // 2 // (6 if t == "fp32" else 1)  # the largest listed one's work
        M = _log(rng, 1, 1 << 17)
        K, N = _width(rng, 64, 8192), _width(rng, 64, 8192)
        while M * K * N * (2 if op == "dense_backward" else 1) > most or M * max(K, N) > 1 << 25:
            M, K, N = _size(M // 2 + 1), _size(max(64, K * 4 // 5)), _size(max(64, N * 4 // 5))
        act, order, bias = rng.choice(ACTS), rng.choice(("io", "oi")), rng.random() < 0.8
        if op == "dense_backward":
            return _grad(None, t, M, K, N, act, bias, p, order, pad)
        return _dense(None, t, M, K, N, act, bias, p, rng.random() < 0.5, rng.random() < 0.3, order, pad)
    d = _width(rng, 64, 8192)
    rows = _log(rng, 1, min(1 << 20, (1 << 26) // d))
    if op == "norm":
        return _norm(None, t, rows, d, pad)
    if op == "norm_grad":
        return _norm_grad(None, t, rows, d, rng.random() < 0.5, pad)
    return _drop(None, t, rows, d, p, rng.random() < 0.5, pad)


# ---- inputs -----------------------------------------------------------------

class _Inputs:
    """A case's inputs from its seed, the same ones for every form of the case."""

    def __init__(self, case, seed):
        self.gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
        self.dt = TYPES[case["type"]]

    def rows(self, n, d, pad=0, scale=1.0, shift=0.0):
        v = torch.randn((n, d + pad), generator=self.gen, device=DEVICE, dtype=torch.float32)
        return v.mul_(scale).add_(shift).to(self.dt)[:, :d]

    def vector(self, d, scale=1.0, shift=0.0):
        return self.rows(1, d, 0, scale, shift).reshape(d)

    def rng(self):
        # (seed, offset) of the dropout's generator: the 64-bit key and the step's number
        return torch.randint(0, 1 << 31, (2,), generator=self.gen, device=DEVICE, dtype=torch.int64)


def _inputs(case, seed):
    i = _Inputs(case, seed)
    s = {"op": case["op"], "dt": i.dt}
    pad = case["pad"]
    if case["op"] in ("dense", "dense_backward"):
        M, K, N = case["M"], case["K"], case["N"]
        s["act"], s["p"] = case["act"], case["p"]
        s["x"] = i.rows(M, K, pad)
        w = i.rows(K, N, 0, K ** -0.5) if case["order"] == "io" else i.rows(N, K, 0, K ** -0.5).t()
        s["w"] = w
        s["b"] = i.vector(N, 0.1) if case["bias"] else None
        s["rng"] = i.rng() if case["p"] > 0 else None
        if case["op"] == "dense":
            s["res"] = i.rows(M, N) if case["residual"] else None
            s["keep_pre"] = case["pre"]
        else:
            s["dy"] = i.rows(M, N, 0, 0.05)
            # the pre-activations that the forward pass left
            s["pre"] = i.rows(M, N) if case["act"] != "none" else None
        return s
    rows, d = case["rows"], case["d"]
    if case["op"] == "dropout":
        s["p"], s["rng"] = case["p"], i.rng()
        s["x"] = i.rows(rows, d, pad)
        s["res"] = i.rows(rows, d) if case["residual"] else None
        return s
    s["x"] = i.rows(rows, d, pad, 1.5, 0.3)
    s["w"], s["b"] = i.vector(d, 0.2, 1.0), i.vector(d, 0.1)
    if case["op"] == "layer_norm_backward":
        s["dy"] = i.rows(rows, d, 0, 0.1)
        s["res"] = i.rows(rows, d, 0, 0.1) if case["residual"] else None
        # the statistics that the forward pass left
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # a call that is repeated on the same buffers: its tensors are checked once
        import paper_2507_01040_amd as cliff
        drop = (s["p"], s["rng"]) if s.get("rng") is not None else None
        if s["op"] == "dense":
            s["plan"] = cliff.dense_plan(s["x"], s["w"], s["b"], act=ACTS.index(s["act"]), dropout=drop,
                                         residual=s["res"], pre=s["keep_pre"])
        elif s["op"] == "dense_backward":
            s["plan"] = cliff.dense_backward_plan(s["dy"], s["x"], s["w"], pre=s["pre"],
                                                  act=ACTS.index(s["act"]), dropout=drop,
                                                  bias=s["b"] is not None)
        elif s["op"] == "layer_norm":
            s["plan"] = cliff.layer_norm_plan(s["x"], s["w"], s["b"], eps=EPS)
        elif s["op"] == "layer_norm_backward":
            s["plan"] = cliff.layer_norm_backward_plan(s["dy"], s["x"], s["mean"], s["rstd"], s["w"],
                                                       dresidual=s["res"])
        else:
            s["plan"] = cliff.dropout_plan(s["x"], s["p"], s["rng"], residual=s["res"])
    return s


# ---- the plain forms ----------------------------------------------------------

_M32 = (1 << 32) - 1


def _mul_hi_lo(a, b):
    # the halves of the 64-bit product of a constant and 32-bit words held in int64
    mid = a * (b >> 16) + ((a * (b & 0xFFFF)) >> 16)
    return mid >> 16, (a * b) & _M32


def _keep(rng, rows, cols, p):
    """Dropout's mask: element (r, c) is kept where word c mod 4 of Philox4x32-7
    (Salmon et al. 2011) with key rng[0] and counter (c div 4, r mod 2^32, r div
    2^32, rng[1]) is at least p 2^32."""
    r = torch.arange(rows, device=DEVICE, dtype=torch.int64)[:, None]
    quads = torch.arange((cols + 3) // 4, device=DEVICE, dtype=torch.int64)[None, :]
    c0, c1, c2, c3 = quads.expand(rows, -1), r & _M32, r >> 32, rng[1] & _M32
    k0, k1 = rng[0] & _M32, (rng[0] >> 32) & _M32
    for _ in range(7):  # the generator's rounds
        h0, l0 = _mul_hi_lo(0xD2511F53, c0)
        h1, l1 = _mul_hi_lo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=-1).reshape(rows, -1)[:, :cols]
    return words >= round(p * 2.0 ** 32)


def _dropped(v, s):
    if s["rng"] is None:
        return v
    keep = _keep(s["rng"], v.shape[0], v.shape[1], s["p"])
    return torch.where(keep, v * (1.0 / (1.0 - s["p"])), torch.zeros_like(v))


def _f(act, v):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 0.5 ** 0.5))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _slope(act, v):
    if act == "relu":
        return (v > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * 0.5 ** 0.5)) + v * torch.exp(-0.5 * v * v) * (2 * math.pi) ** -0.5
    g = 1.0 / (1.0 + torch.exp(-v))
    return g * (1.0 + v * (1.0 - g))


def _plain(s):
    dt, x = s["dt"], s["x"].float()
    if s["op"] == "dense":
        pre = x @ s["w"].float()
        if s["b"] is not None:
            pre = pre + s["b"].float()
        y = _dropped(_f(s["act"], pre), s)
        if s["res"] is not None:
            y = y + s["res"].float()
        return (y.to(dt), pre.to(dt)) if s["keep_pre"] else y.to(dt)
    if s["op"] == "dense_backward":
        g = s["dy"].float()
        if s["act"] != "none":
            g = g * _slope(s["act"], s["pre"].float())
        g = _dropped(g, s)
        dx, dw = g @ s["w"].float().t(), x.t() @ g
        return (dx.to(dt), dw.to(dt), g.sum(0).to(dt)) if s["b"] is not None else (dx.to(dt), dw.to(dt))
    if s["op"] == "layer_norm":
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        return (x * rstd[:, None] * s["w"].float() + s["b"].float()).to(dt), mean, rstd
    if s["op"] == "layer_norm_backward":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        h = (x - s["mean"][:, None]) * rstd
        q = dy * s["w"].float()
        dx = rstd * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
        if s["res"] is not None:
            dx = dx + s["res"].float()
        return dx.to(dt), (dy * h).sum(0).to(dt), dy.sum(0).to(dt)
    y = _dropped(x, s)
    return (y + s["res"].float() if s["res"] is not None else y).to(dt)


def run(s):
    return s["plan"]() if own else _plain(s)


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    e = 4 if case["type"] == "fp32" else 2
    if case["op"] == "dense":
        M, K, N = case["M"], case["K"], case["N"]
        n = M * K + K * N + N * case["bias"] + M * N * (1 + case["residual"] + case["pre"])
        return {"bytes": n * e, "flops": 2 * M * N * K + 4 * M * N}
    if case["op"] == "dense_backward":
        M, K, N = case["M"], case["K"], case["N"]
        n = M * N * (1 + (case["act"] != "none")) + 2 * M * K + 2 * K * N + N * case["bias"]
        return {"bytes": n * e, "flops": 4 * M * N * K + 4 * M * N}
    n = case["rows"] * case["d"]
    if case["op"] == "layer_norm":
        return {"bytes": (2 * n + 2 * case["d"]) * e + 8 * case["rows"], "flops": 8 * n}
    if case["op"] == "layer_norm_backward":
        return {"bytes": ((3 + case["residual"]) * n + 3 * case["d"]) * e + 8 * case["rows"],
                "flops": 16 * n}
    return {"bytes": (2 + case["residual"]) * n * e, "flops": 2 * n}


# ---- the definitions in 64 bits ------------------------------------------------------

def _exact_mask(key, offset, rows, cols, p):
    # the same generator from its definition, on 16-bit limbs: product (h, l) of a
    # 32-bit constant m and a word
    dev = DEVICE

    def product(m, word):
        m1, m0 = m >> 16, m & 0xFFFF
        w1, w0 = word.div(65536, rounding_mode="floor"), word.remainder(65536)
        low = m0 * w0
        cross = m1 * w0 + low.div(65536, rounding_mode="floor")
        cross2 = m0 * w1 + cross.remainder(65536)
        high = m1 * w1 + cross.div(65536, rounding_mode="floor") + cross2.div(65536, rounding_mode="floor")
        return high, cross2.remainder(65536) * 65536 + low.remainder(65536)

    two32 = 2 ** 32
    nq = -(-cols // 4)
    row = torch.arange(rows, device=dev).repeat_interleave(nq)
    state = [torch.arange(nq, device=dev).repeat(rows), row.remainder(two32),
             row.div(two32, rounding_mode="floor"), torch.full_like(row, offset % two32)]
    key = [key % two32, key // two32 % two32]
    for step in range(7):
        a, b = product(0xD2511F53, state[0]), product(0xCD9E8D57, state[2])
        ks = [(key[0] + step * 0x9E3779B9) % two32, (key[1] + step * 0xBB67AE85) % two32]
        state = [b[0].bitwise_xor(state[1]).bitwise_xor(ks[0]), b[1],
                 a[0].bitwise_xor(state[3]).bitwise_xor(ks[1]), a[1]]
    out = torch.empty((rows, 4 * nq), device=dev, dtype=torch.bool)
    for word in range(4):
        out[:, word::4] = (state[word] >= int(p * two32 + 0.5)).view(rows, nq)
    return out[:, :cols]


def exact(case, seed):
    s = _inputs(case, seed)
    d = lambda t: None if t is None else t.double()  # noqa: E731
    mask = None
    if s.get("rng") is not None:
        key, offset = s["rng"].tolist()
        shape = (case["M"], case["N"]) if "M" in case else (case["rows"], case["d"])
        mask = _exact_mask(key, offset, *shape, case["p"]).double() / (1 - case["p"])
    x = d(s["x"])
    phi = torch.special.ndtr
    if case["op"] == "dense":
        pre = torch.mm(x, d(s["w"]).contiguous())
        if s["b"] is not None:
            pre += d(s["b"])
        act = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * phi(v),
               "silu": lambda v: v * torch.sigmoid(v)}[case["act"]]
        y = act(pre)
        if mask is not None:
            y = y * mask
        if s["res"] is not None:
            y = y + d(s["res"])
        return (y, pre) if case["pre"] else y
    if case["op"] == "dense_backward":
        g = d(s["dy"])
        v = d(s["pre"])
        if case["act"] == "relu":
            g = g.masked_fill(v <= 0, 0.0)
        elif case["act"] == "gelu":
            g = g * (phi(v) + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi))
        elif case["act"] == "silu":
            sg = torch.sigmoid(v)
            g = g * (sg + v * sg * (1 - sg))
        if mask is not None:
            g = g * mask
        dx = torch.mm(g, d(s["w"]).t().contiguous())
        dw = torch.mm(x.t().contiguous(), g)
        return (dx, dw, g.sum(dim=0)) if case["bias"] else (dx, dw)
    if case["op"] == "layer_norm":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        return (x - mean.unsqueeze(1)) * rstd.unsqueeze(1) * d(s["w"]) + d(s["b"]), mean, rstd
    if case["op"] == "layer_norm_backward":
        dy, i = d(s["dy"]), d(s["rstd"]).unsqueeze(1)
        h = (x - d(s["mean"]).unsqueeze(1)) * i
        q = dy * d(s["w"])
        n = case["d"]
        dx = (q - q.sum(1, keepdim=True) / n - h * ((q * h).sum(1, keepdim=True) / n)) * i
        if s["res"] is not None:
            dx = dx + d(s["res"])
        return dx, torch.sum(dy * h, 0), torch.sum(dy, 0)
    y = x * mask
    return y + d(s["res"]) if s["res"] is not None else y
