"""The operators of a residual feed-forward block in 8 bits that are measured:
rows quantized to 8-bit integers and back, the dense layer of 8-bit integers with
a scale for each token and channel, the dense layer's gradient from 8-bit
checkpoints of its input and pre-activations, and the norms after and before a
block fused with its gate and the scaled residual, with their gradient.

Rows are tokens, or the flattened multivectors (C * N_B features) between two
Clifford linear layers.  Sizes are those of the repository's linear layers
(32 channels of 4 blades: 128 features, up to 2^20 rows) and generic ones of
feed-forward parts; `draw` spreads over the same ranges: one row to many, odd
widths, padded rows, every type, activation, norm and gate.

The plain forms compute in float32 and round once (quantized values in float64,
where a quotient next to the border of two integers decides).  `exact` computes
in float64.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")  # in the order of the library's constants
EPS = 1e-5
GROUP = 128  # features that share a checkpoint's scale


def _quant(name, t, rows, d, grouped, pad=0):
    # grouped: a scale for each 128 features of a row, else one for the row; pad:
    # elements between the rows of x beyond its width
    c = {"op": "quantize", "type": t, "rows": rows, "d": d, "grouped": grouped, "pad": pad}
    return dict(c, name=name) if name else c


def _int8(name, t, M, K, N, act, bias=True, residual=False, pad=0):
    c = {"op": "dense_int8", "type": t, "M": M, "K": K, "N": N, "act": act, "bias": bias,
         "residual": residual, "pad": pad}
    return dict(c, name=name) if name else c


def _grad(name, t, M, K, N, act, bias=True, p=0.0, order="io", grouped=True, pad=0):
    # order: the weight is [in, out] ("io") or a transposed view of [out, in] ("oi")
    c = {"op": "dense_backward_int8", "type": t, "M": M, "K": K, "N": N, "act": act, "bias": bias,
         "p": p, "order": order, "grouped": grouped, "pad": pad}
    return dict(c, name=name) if name else c


def _norm(name, t, rows, d, groups, scale=1.0, after=True, before=True, rms=False, pad=0):
    # groups: 0, no gate; 1, a gate for each feature; more, one for each group of rows as well
    c = {"op": "block_norm", "type": t, "rows": rows, "d": d, "groups": groups, "scale": scale,
         "after": after, "before": before, "rms": rms, "pad": pad}
    return dict(c, name=name) if name else c


def _norm_grad(name, t, rows, d, groups, scale=1.0, after=True, before=True, rms=False, pad=0):
    c = _norm(name, t, rows, d, groups, scale, after, before, rms, pad)
    c["op"] = "block_norm_backward"
    return c


def listed():
    return [
        # the rows of a few tokens for the next 8-bit product while serving: latency
        _quant("quantize_few_rows", "bf16", 4, 4096, False),
        # a layer's input kept for the backward pass, and read back
        _quant("checkpoint_large", "bf16", 16384, 4096, True),
        # one token through a block's first layer while serving: the weight's read
        _int8("int8_one_row", "bf16", 1, 4096, 8192, "silu"),
        # a small batch of tokens while serving, the second layer with its residual
        _int8("int8_few_rows", "fp16", 24, 8192, 4096, "none", residual=True),
        # a ragged batch: no size a multiple of a vector, rows of x padded
        _int8("int8_odd", "fp16", 1003, 777, 1531, "gelu", residual=True, pad=5),
        # a large batch, as for prompts read while serving
        _int8("int8_large", "bf16", 4096, 4096, 8192, "gelu"),
        # the gradient of an ordinary feed-forward layer in training
        _grad("grad_int8", "bf16", 8192, 2048, 2048, "gelu", p=0.1),
        # the gradient of the framework's rows: a long sum over rows, few weights
        _grad("grad_int8_multivectors", "fp32", 1 << 16, 128, 512, "silu"),
        # the norms around a block for a few tokens while serving: latency
        _norm("block_norm_few_rows", "bf16", 4, 4096, 1, rms=True),
        # the norms around a block of the framework's rows, a gate for each of 64 fields
        _norm("block_norm_multivectors", "fp32", 1 << 19, 128, 64),
        # the norms' gradient in training, gate and residual scale included
        _norm_grad("block_norm_grad", "bf16", 16384, 4096, 1, scale=0.5),
        # the gradient on a ragged batch, conditioned gates, padded rows
        _norm_grad("block_norm_grad_odd", "fp16", 1001, 777, 7, rms=True, pad=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    # an odd width half of the time, else a power of two or 5/4 of one
    w = _log(rng, lo, hi)
    if rng.random() < 0.5:
        return w | 1
    w = 1 << (w.bit_length() - 1)
    return min(hi, w * rng.choice((4, 4, 5)) // 4)


def draw(rng):
    t = rng.choice(("fp32", "bf16", "fp16"))
    pad = rng.choice((0, 0, rng.randint(1, 16), 64))
    op = rng.choice(("quantize", "dense_int8", "dense_int8", "dense_backward_int8", "block_norm",
                     "block_norm_backward"))
    if op.startswith("dense"):
        # the work of the largest listed case of the operator
        most = 4096 * 4096 * 8192 if op == "dense_int8" else 8192 * 2048 * 2048 // (6 if t == "fp32" else 1)
        M = _log(rng, 1, 1 << 17)
        K, N = _width(rng, 64, 8192), _width(rng, 64, 8192)
        while M * K * N > most or M * max(K, N) > 1 << 25:
            M, K, N = M // 2 + 1, max(64, K * 4 // 5), max(64, N * 4 // 5)
        act, bias = rng.choice(ACTS), rng.random() < 0.8
        if op == "dense_int8":
            return _int8(None, t, M, K, N, act, bias, rng.random() < 0.5, pad)
        p = rng.choice((0.0, 0.1, round(rng.uniform(0.05, 0.6), 3)))
        return _grad(None, t, M, K, N, act, bias, p, rng.choice(("io", "oi")), rng.random() < 0.7, pad)
    d = _width(rng, 64, 8192)
    rows = _log(rng, 1, min(1 << 20, (1 << 26) // d))
    if op == "quantize":
        return _quant(None, t, rows, d, rng.random() < 0.5, pad)
    groups = rng.choice((0, 1, 1, rng.randint(2, 64)))
    if groups > 1:
        rows = max(1, rows // groups) * groups
    after, before = rng.choice(((True, True), (True, True), (True, False), (False, True)))
    make = _norm if op == "block_norm" else _norm_grad
    return make(None, t, rows, d, groups, rng.choice((1.0, 1.0, 0.5, 2.5)), after, before,
                rng.random() < 0.5, pad)


# ---- inputs -----------------------------------------------------------------

class _Inputs:
    """A case's inputs from its seed, the same ones for every form of the case."""

    def __init__(self, case, seed):
        self.gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
        self.dt = TYPES[case["type"]]

    def floats(self, n, d):
        return torch.randn((n, d), generator=self.gen, device=DEVICE, dtype=torch.float32)

    def rows(self, n, d, pad=0, scale=1.0, shift=0.0):
        return self.floats(n, d + pad).mul_(scale).add_(shift).to(self.dt)[:, :d]

    def features(self, n, d, pad=0):
        # activations: some features are several times as large as others
        return (self.floats(n, d + pad) * torch.exp(0.5 * self.floats(1, d + pad))).to(self.dt)[:, :d]

    def vector(self, d, scale=1.0, shift=0.0):
        return self.rows(1, d, 0, scale, shift).reshape(d)

    def rng(self):
        # (seed, offset) of the dropout's generator: the 64-bit key and the step's number
        return torch.randint(0, 1 << 31, (2,), generator=self.gen, device=DEVICE, dtype=torch.int64)


def _eight(x, grouped, pad=0):
    """(integers, scales) of a matrix x: what an earlier call left."""
    rows, d = x.shape
    n = -(-d // GROUP) if grouped else 1
    wide = torch.zeros((rows, n * GROUP if grouped else d), device=DEVICE, dtype=torch.float32)
    wide[:, :d] = x.float()
    wide = wide.reshape(rows, n, -1)
    scale = torch.clamp(wide.abs().amax(2) / 127.0, min=2.0 ** -126)
    q = torch.round(wide / scale[:, :, None]).reshape(rows, -1)
    out = torch.zeros((rows, d + pad), device=DEVICE, dtype=torch.int8)
    out[:, :d] = q[:, :d].to(torch.int8)
    return out[:, :d], scale


def _inputs(case, seed):
    i = _Inputs(case, seed)
    s = {"op": case["op"], "dt": i.dt}
    pad = case["pad"]
    if case["op"] == "quantize":
        s["grouped"] = case["grouped"]
        s["x"] = i.features(case["rows"], case["d"], pad)
        return s
    if case["op"] == "dense_int8":
        M, K, N = case["M"], case["K"], case["N"]
        s["act"] = case["act"]
        s["x"], s["xs"] = _eight(i.features(M, K), False, pad)
        s["w"], s["ws"] = _eight(i.rows(N, K, 0, K ** -0.5), False)  # [out, in], a scale for each output
        s["b"] = i.vector(N, 0.1) if case["bias"] else None
        s["res"] = i.rows(M, N) if case["residual"] else None
        return s
    if case["op"] == "dense_backward_int8":
        M, K, N = case["M"], case["K"], case["N"]
        s["act"], s["p"], s["bias"] = case["act"], case["p"], case["bias"]
        s["x"], s["xs"] = _eight(i.features(M, K), case["grouped"], pad)
        s["w"] = i.rows(K, N, 0, K ** -0.5) if case["order"] == "io" else i.rows(N, K, 0, K ** -0.5).t()
        s["dy"] = i.rows(M, N, 0, 0.05)
        # the pre-activations that the forward pass left
        s["pre"], s["ps"] = _eight(i.rows(M, N), case["grouped"]) if case["act"] != "none" else (None, None)
        s["rng"] = i.rng() if case["p"] > 0 else None
        return s
    rows, d, groups = case["rows"], case["d"], case["groups"]
    for k in ("scale", "after", "before", "rms"):
        s[k] = case[k]
    s["x"] = i.rows(rows, d, pad, 1.5, 0.3)
    s["w"], s["b"] = (i.vector(d, 0.2, 1.0), i.vector(d, 0.1)) if case["after"] else (None, None)
    s["nw"], s["nb"] = (i.vector(d, 0.2, 1.0), i.vector(d, 0.1)) if case["before"] else (None, None)
    if case["rms"]:
        s["b"] = s["nb"] = None
    s["gate"] = None
    if groups:
        g = i.rows(groups, d, 0, 0.3, 0.6)
        s["gate"] = g.reshape(d) if groups == 1 else g
    if case["op"] == "block_norm":
        s["res"] = i.rows(rows, d, 0, 2.0)
        return s
    # what the forward pass left: the new residual row, and the statistics
    s["out"] = i.rows(rows, d, 0, 2.0, 0.1)
    s["stats"] = torch.cat([_statistics(s[k].float(), case["rms"]) for k in ("x", "out")])
    s["dout"] = i.rows(rows, d, 0, 0.1)
    s["dnormed"] = i.rows(rows, d, 0, 0.1) if case["before"] else None
    return s


def _statistics(v, rms):
    mean = torch.zeros_like(v[:, 0]) if rms else v.mean(1)
    return torch.stack([mean, ((v - mean[:, None]) ** 2).mean(1).add(EPS).rsqrt()])


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # a call that is repeated on the same buffers: its tensors are checked once
        import paper_2507_01040_amd as cliff
        drop = (s["p"], s["rng"]) if s.get("rng") is not None else None
        if s["op"] == "quantize":
            s["plan"] = cliff.quantize_plan(s["x"], group=GROUP if s["grouped"] else None)
            s["back"] = cliff.dequantize_plan(*s["plan"].out, dtype=s["dt"])
        elif s["op"] == "dense_int8":
            s["plan"] = cliff.dense_int8_plan(s["x"], s["xs"], s["w"].t(), s["ws"], s["b"],
                                              act=ACTS.index(s["act"]), residual=s["res"], dtype=s["dt"])
        elif s["op"] == "dense_backward_int8":
            s["plan"] = cliff.dense_backward_int8_plan(s["dy"], s["x"], s["xs"], s["w"], pre=s["pre"],
                                                       pre_scale=s["ps"], act=ACTS.index(s["act"]),
                                                       dropout=drop, bias=s["bias"])
        elif s["op"] == "block_norm":
            s["plan"] = cliff.block_norm_plan(s["x"], s["res"], gate=s["gate"], scale=s["scale"],
                                              weight=s["w"], bias=s["b"], next_weight=s["nw"],
                                              next_bias=s["nb"], after=s["after"], before=s["before"],
                                              rms=s["rms"], eps=EPS)
        else:
            s["plan"] = cliff.block_norm_backward_plan(s["dout"], s["dnormed"], s["x"], s["out"], s["stats"],
                                                       gate=s["gate"], scale=s["scale"], weight=s["w"],
                                                       bias=s["b"], next_weight=s["nw"], next_bias=s["nb"],
                                                       after=s["after"], rms=s["rms"])
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


def _spread(scale, d):
    # a row's scales, one for each of its d features
    return scale if scale.shape[1] == 1 else scale.repeat_interleave(GROUP, 1)[:, :d]


def _plain(s):
    dt = s["dt"]
    if s["op"] == "quantize":
        x = s["x"].float()
        rows, d = x.shape
        if s["grouped"]:
            n = -(-d // GROUP)
            wide = torch.zeros((rows, n * GROUP), device=x.device, dtype=x.dtype)
            wide[:, :d] = x
            most = wide.abs().reshape(rows, n, GROUP).amax(2)
        else:
            most = x.abs().amax(1, keepdim=True)
        scale = torch.clamp((most.double() / 127.0).float(), min=2.0 ** -126)
        each = _spread(scale, d)
        q = torch.round(x.double() / each).float()
        return (q * each).to(dt), scale
    if s["op"] == "dense_int8":
        pre = (s["x"].float() @ s["w"].float().t()) * s["xs"] * s["ws"].reshape(1, -1)
        if s["b"] is not None:
            pre = pre + s["b"].float()
        y = _f(s["act"], pre)
        return (y if s["res"] is None else y + s["res"].float()).to(dt)
    if s["op"] == "dense_backward_int8":
        x = s["x"].float() * _spread(s["xs"], s["x"].shape[1])
        g = s["dy"].float()
        if s["act"] != "none":
            g = g * _slope(s["act"], s["pre"].float() * _spread(s["ps"], g.shape[1]))
        if s["rng"] is not None:
            keep = _keep(s["rng"], g.shape[0], g.shape[1], s["p"])
            g = torch.where(keep, g * (1.0 / (1.0 - s["p"])), torch.zeros_like(g))
        dx, dw = g @ s["w"].float().t(), x.t() @ g
        return (dx.to(dt), dw.to(dt), g.sum(0).to(dt)) if s["bias"] else (dx.to(dt), dw.to(dt))
    x = s["x"].float()
    if s["op"] == "block_norm":
        stats = []

        def norm(v, w, b):
            st = _statistics(v, s["rms"])
            stats.append(st)
            v = (v - st[0][:, None]) * st[1][:, None]
            v = v if w is None else v * w.float()
            return v if b is None else v + b.float()

        h = norm(x, s["w"], s["b"]) if s["after"] else x
        if s["gate"] is not None:
            g = s["gate"].float().reshape(-1, x.shape[1])[:, None, :]  # for each group's rows
            h = (h.reshape(g.shape[0], -1, x.shape[1]) * g).reshape(x.shape)
        out = s["scale"] * s["res"].float() + h
        if s["before"]:
            return out.to(dt), norm(out, s["nw"], s["nb"]).to(dt), torch.cat(stats)
        return out.to(dt), torch.cat(stats)
    m1, r1, m2, r2 = (v[:, None] for v in s["stats"])

    def through(q, h, r):
        # the gradient of a norm's input, of normed values h
        u = q if s["rms"] else q - q.mean(1, keepdim=True)
        return r * (u - h * (q * h).mean(1, keepdim=True))

    t = s["dout"].float()
    grads = {}
    if s["before"]:
        dn, h = s["dnormed"].float(), (s["out"].float() - m2) * r2
        t = t + through(dn * s["nw"].float(), h, r2)
        grads["nw"], grads["nb"] = (dn * h).sum(0), dn.sum(0)
    h = (x - m1) * r1 if s["after"] else x
    v = h
    if s["after"]:
        v = v * s["w"].float()
        v = v if s["b"] is None else v + s["b"].float()
    u = t
    if s["gate"] is not None:
        g = s["gate"].float().reshape(-1, x.shape[1])[:, None, :]  # for each group's rows
        per_group = t.reshape(g.shape[0], -1, x.shape[1])
        grads["gate"] = (per_group * v.reshape(per_group.shape)).sum(1).reshape(s["gate"].shape)
        u = (per_group * g).reshape(x.shape)
    if s["after"]:
        grads["w"], grads["b"] = (u * h).sum(0), u.sum(0)
        dx = through(u * s["w"].float(), h, r1)
    else:
        dx = u
    outs = [dx, s["scale"] * t] + [grads[k] for k in ("gate", "w", "b", "nw", "nb") if s[k] is not None]
    return tuple(v.to(dt) for v in outs)


def run(s):
    if not own:
        return _plain(s)
    out = s["plan"]()
    if s["op"] == "quantize":
        return s["back"](), out[1]
    if s["op"] == "block_norm":
        # the rows of the statistics that belong to a norm of the call
        used = out[-1][0 if s["after"] else 2:4 if s["before"] else 2]
        return (*out[:-1], used)
    if s["op"] == "block_norm_backward":
        return tuple(v for v in out if v is not None)
    return out


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    e = 4 if case["type"] == "fp32" else 2
    if case["op"] == "quantize":
        n = case["rows"] * case["d"]
        scales = case["rows"] * (-(-case["d"] // GROUP) if case["grouped"] else 1)
        return {"bytes": 2 * n * e + 4 * scales, "flops": 4 * n}
    if case["op"] == "dense_int8":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K + K * N + 4 * (M + N) + (N * case["bias"] + M * N * (1 + case["residual"])) * e,
                "flops": 2 * M * N * K + 4 * M * N}
    if case["op"] == "dense_backward_int8":
        M, K, N = case["M"], case["K"], case["N"]
        act = case["act"] != "none"
        scales = M * (-(-K // GROUP) + act * -(-N // GROUP) if case["grouped"] else 1 + act)
        n = M * N + M * K + 2 * K * N + N * case["bias"]
        return {"bytes": n * e + M * K + M * N * act + 4 * scales, "flops": 4 * M * N * K + 4 * M * N}
    n, vectors = case["rows"] * case["d"], case["d"] * (case["groups"] + case["after"] + case["before"])
    if case["op"] == "block_norm":
        return {"bytes": (n * (3 + case["before"]) + vectors) * e + 8 * case["rows"] * (case["after"] + case["before"]),
                "flops": n * (4 + 8 * (case["after"] + case["before"]))}
    # x is read for a norm or a gate, the new row for the norm before the next block
    reads = 1 + 2 * case["before"] + (case["after"] or case["groups"] > 0)
    return {"bytes": (n * (reads + 2) + 2 * vectors) * e + 8 * case["rows"] * (case["after"] + case["before"]),
            "flops": n * (4 + 16 * (case["after"] + case["before"]))}


# ---- the definitions in 64 bits ------------------------------------------------------

def _exact_mask(key, offset, rows, cols, p):
    # the same generator from its definition, on 16-bit limbs: product (h, l) of a
    # 32-bit constant m and a word
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
    row = torch.arange(rows, device=DEVICE).repeat_interleave(nq)
    state = [torch.arange(nq, device=DEVICE).repeat(rows), row.remainder(two32),
             row.div(two32, rounding_mode="floor"), torch.full_like(row, offset % two32)]
    key = [key % two32, key // two32 % two32]
    for step in range(7):
        a, b = product(0xD2511F53, state[0]), product(0xCD9E8D57, state[2])
        ks = [(key[0] + step * 0x9E3779B9) % two32, (key[1] + step * 0xBB67AE85) % two32]
        state = [b[0].bitwise_xor(state[1]).bitwise_xor(ks[0]), b[1],
                 a[0].bitwise_xor(state[3]).bitwise_xor(ks[1]), a[1]]
    out = torch.empty((rows, 4 * nq), device=DEVICE, dtype=torch.bool)
    for word in range(4):
        out[:, word::4] = (state[word] >= int(p * two32 + 0.5)).view(rows, nq)
    return out[:, :cols]


def _exact_values(q, scale):
    # the numbers that integers and their scales stand for
    parts = [q[:, c:c + GROUP] for c in range(0, q.shape[1], GROUP)] if scale.shape[1] > 1 else [q]
    return torch.cat([p.double() * scale[:, i:i + 1].double() for i, p in enumerate(parts)], dim=1)


def _exact_norm(v, rms, weight, bias):
    mean = torch.zeros(v.shape[0], device=v.device, dtype=v.dtype) if rms else v.sum(1) / v.shape[1]
    centred = v - mean.unsqueeze(1)
    rstd = (centred.square().sum(1) / v.shape[1] + EPS).pow(-0.5)
    y = centred * rstd.unsqueeze(1)
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, [mean, rstd]


def _exact_gate(s, like):
    if s["gate"] is None:
        return torch.ones_like(like)
    g = s["gate"].double().reshape(-1, like.shape[1])
    which = torch.arange(like.shape[0], device=like.device).div(like.shape[0] // g.shape[0], rounding_mode="floor")
    return g[which]


def exact(case, seed):
    s = _inputs(case, seed)
    phi = torch.special.ndtr
    if case["op"] == "quantize":
        x = s["x"].double()
        width = GROUP if case["grouped"] else case["d"]
        values, scales = [], []
        for c in range(0, case["d"], width):
            part = x[:, c:c + width]
            most = torch.maximum(part.amax(1), -part.amin(1))
            scale = (most / 127).float().double().clamp(min=2.0 ** -126).unsqueeze(1)
            scales.append(scale)
            values.append(torch.round(part / scale) * scale)
        return torch.cat(values, 1), torch.cat(scales, 1)
    if case["op"] == "dense_int8":
        pre = torch.mm(_exact_values(s["x"], s["xs"]), _exact_values(s["w"], s["ws"]).t().contiguous())
        if s["b"] is not None:
            pre += s["b"].double()
        act = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * phi(v),
               "silu": lambda v: v * torch.sigmoid(v)}[case["act"]]
        y = act(pre)
        return y if s["res"] is None else y + s["res"].double()
    if case["op"] == "dense_backward_int8":
        g = s["dy"].double()
        if case["act"] != "none":
            v = _exact_values(s["pre"], s["ps"])
            if case["act"] == "relu":
                g = g.masked_fill(v <= 0, 0.0)
            elif case["act"] == "gelu":
                g = g * (phi(v) + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi))
            else:
                sg = torch.sigmoid(v)
                g = g * (sg + v * sg * (1 - sg))
        if s["rng"] is not None:
            key, offset = s["rng"].tolist()
            g = g * (_exact_mask(key, offset, case["M"], case["N"], case["p"]).double() / (1 - case["p"]))
        dx = torch.mm(g, s["w"].double().t().contiguous())
        dw = torch.mm(_exact_values(s["x"], s["xs"]).t().contiguous(), g)
        return (dx, dw, g.sum(dim=0)) if case["bias"] else (dx, dw)
    x = s["x"].double()
    gate = _exact_gate(s, x)
    if case["op"] == "block_norm":
        h, stats = _exact_norm(x, s["rms"], s["w"], s["b"]) if case["after"] else (x, [])
        out = s["res"].double() * case["scale"] + h * gate
        if not case["before"]:
            return out, torch.stack(stats)
        normed, more = _exact_norm(out, s["rms"], s["nw"], s["nb"])
        return out, normed, torch.stack(stats + more)
    stats = s["stats"].double().unsqueeze(2)
    n = case["d"]

    def back(q, h, rstd):
        dot = torch.sum(q * h, 1, keepdim=True) / n
        shift = 0.0 if case["rms"] else torch.sum(q, 1, keepdim=True) / n
        return (q - shift - h * dot) * rstd

    t, grads = s["dout"].double(), {}
    if case["before"]:
        dn, h2 = s["dnormed"].double(), (s["out"].double() - stats[2]) * stats[3]
        grads["nw"], grads["nb"] = torch.sum(dn * h2, 0), torch.sum(dn, 0)
        t = t + back(dn * s["nw"].double(), h2, stats[3])
    if case["after"]:
        h1 = (x - stats[0]) * stats[1]
        value = h1 * s["w"].double() + (0.0 if s["b"] is None else s["b"].double())
        grads["w"], grads["b"] = torch.sum(t * gate * h1, 0), torch.sum(t * gate, 0)
        dx = back(t * gate * s["w"].double(), h1, stats[1])
    else:
        value, dx = x, t * gate
    if s["gate"] is not None:
        each = torch.zeros((max(1, case["groups"]), n), device=x.device, dtype=x.dtype)
        per = case["rows"] // case["groups"]
        for i in range(case["groups"]):
            each[i] = torch.sum(t[i * per:(i + 1) * per] * value[i * per:(i + 1) * per], 0)
        grads["gate"] = each.reshape(s["gate"].shape)
    return tuple([dx, t * case["scale"]] + [grads[k] for k in ("gate", "w", "b", "nw", "nb") if s[k] is not None])
