"""Plain implementations in 64 bits of the 8-bit operators and the block norm, on the
CPU, and the error bounds of their tests, derived as in ff_oracle.py (sums of
integers are exact; a sum's terms that are not exact themselves add their own
errors)."""
import numpy as np
import torch

import ff_oracle as O
from ff_oracle import COST, LAMBDA, SLOPE, TINY, U, UNIT

GROUP = 128


def _d(t):
    return None if t is None else t.detach().cpu().double()


def _out(v, e, dtype):
    u, t = UNIT[dtype], TINY[dtype]
    return v, e * (1 + u) + 2 * u * v.abs() + t


def quantize(x, group):
    """(q, scale), exactly: float64 q, float32 scale [rows, groups]."""
    x = _d(x)
    rows, d = x.shape
    step = group or max(d, 1)
    qs, scales = [], []
    for c in range(0, d, step):
        part = x[:, c:c + step]
        finite = torch.isfinite(part).all(1)
        most = torch.where(finite, part.abs().nan_to_num(0, 0, 0).amax(1), torch.zeros(rows, dtype=torch.float64))
        # (a float64 quotient of a float32 and 127 is no tie of two float32)
        scale = (most / 127).float().clamp(min=2.0 ** -126)
        q = torch.from_numpy(np.rint((part / scale.double()[:, None]).numpy()))
        qs.append(torch.where(finite[:, None], q, torch.zeros_like(q)))
        scales.append(torch.where(finite, scale, torch.full_like(scale, float("nan"))))
    return torch.cat(qs, 1), torch.stack(scales, 1)


def values(q, scale):
    """What integers and scales [rows, groups] stand for."""
    q, scale = _d(q).reshape(-1, q.shape[-1]), _d(scale)
    each = scale if scale.shape[1] == 1 else scale.repeat_interleave(GROUP, 1)[:, :q.shape[1]]
    return q * each


def dequantize(q, scale, dtype):
    v = values(q, scale)
    return _out(v, U * v.abs(), dtype)


def dense_int8(x, xs, w, ws, b, a, res, dtype):
    """w [K, N]."""
    p = (_d(x) @ _d(w)) * _d(xs) * _d(ws).reshape(1, -1)
    b = _d(b) if b is not None else torch.zeros(1, dtype=torch.float64)
    pre, e = p + b, 4 * U * (p.abs() + b.abs())
    f = O.act(a, pre)
    y, ey = f, SLOPE * e + COST * U * (f.abs() + (pre.abs() if a else 0))
    if res is not None:
        y, ey = y + _d(res), ey + 2 * U * _d(res).abs()
    return _out(y, ey, dtype)


def dense_backward_int8(dy, x, xs, w, pre, ps, a, dropout, dtype):
    """((dx, bound), (dw, bound), (db, bound)): those of the gradient at the values
    that x and pre stand for, and x's rounding to its type."""
    xv = values(x, xs)
    dx, dw, db = O.dense_backward(dy, xv, w, values(pre, ps) if a else None, a, dropout, dtype)
    g = _d(dy).abs() * (SLOPE if a else 1)
    if dropout is not None:
        g = g * O.mask(dropout, *g.shape)
    u = UNIT[dtype]
    ex = (U + u) * xv.abs() + TINY[dtype]
    return dx, (dw[0], dw[1] + (ex.t() @ g) * (1 + 4 * u)), db


class _Norm:
    """A norm of rows v with errors e: normed values h with errors eh."""

    def __init__(self, v, e, rms, eps):
        d = v.shape[1]
        s = (LAMBDA * d ** 0.5 + COST) * U
        self.mean = torch.zeros(v.shape[0], dtype=torch.float64) if rms else v.mean(1)
        self.em = torch.zeros_like(self.mean) if rms else e.mean(1) + s * v.abs().mean(1)
        c, m = v - self.mean[:, None], self.em[:, None]
        var = (c * c).mean(1)
        # the mean's own error moves the sum of squares in second order only
        ev = (2 * c.abs() * e + (e + m + U * v.abs()) ** 2 + 2 * U * c.abs() * v.abs()).mean(1)
        self.rstd = (var + eps) ** -0.5
        self.er = self.rstd * (0.5 * (ev + s * var + 2 * U * eps) * self.rstd ** 2 + 4 * U)
        r, er = self.rstd[:, None], self.er[:, None]
        self.h = c * r
        self.eh = (e + m + U * v.abs()) * (r + er) + c.abs() * er + 4 * U * self.h.abs()

    def affine(self, w, b):
        h, e = self.h, self.eh
        if w is not None:
            h = h * _d(w)
            e = e * _d(w).abs() + 2 * U * h.abs()
        if b is not None:
            e = e + 2 * U * (h.abs() + _d(b).abs())
            h = h + _d(b)
        return h, e


def _gate(gate, rows, d):
    if gate is None:
        return torch.ones(rows, d, dtype=torch.float64)
    g = _d(gate).reshape(-1, d)
    return g.repeat_interleave(rows // g.shape[0], 0)


def block_norm(x, res, gate, scale, w, b, nw, nb, after, before, rms, eps, dtype):
    """(out, normed or None, stats [4 or 2 rows]), each with its bound."""
    v = _d(x)
    e = torch.zeros_like(v)
    stats = []
    if after:
        n = _Norm(v, e, rms, eps)
        stats += [(n.mean, n.em + 1e-37), (n.rstd, n.er + 1e-37)]
        v, e = n.affine(w, b)
    g = _gate(gate, *v.shape)
    r = scale * _d(res)
    e = e * g.abs() + 3 * U * ((v * g).abs() + r.abs())
    v = v * g + r
    out = _out(v, e, dtype)
    normed = None
    if before:
        n = _Norm(v, e, rms, eps)
        stats += [(n.mean, n.em + 1e-37), (n.rstd, n.er + 1e-37)]
        normed = _out(*n.affine(nw, nb), dtype)
    return out, normed, stats


def block_norm_backward(dout, dnormed, x, out, stats, gate, scale, w, b, nw, after, rms, dtype):
    """{name: (value, bound)} of BlockNormGradients, for the given statistics."""
    like = dnormed if dnormed is not None else dout
    R, d = like.shape
    stats = _d(stats)
    s, sr = (LAMBDA * d ** 0.5 + COST) * U, (LAMBDA * max(R, 1) ** 0.5 + COST) * U

    def normed(v, k):
        v, m, i = _d(v), stats[k][:, None], stats[k + 1][:, None]
        h = (v - m) * i
        return h, 4 * U * (h.abs() + (v.abs() + m.abs()) * i), i

    def through(q, eq, h, eh, i):
        mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
        m, em = (0 * mean(q), 0) if rms else (mean(q), mean(eq) + s * mean(q.abs()))
        mh = mean(q * h)
        emh = mean(eq * h.abs() + (q.abs() + eq) * eh) + s * mean((q * h).abs())
        o = i * (q - m - h * mh)
        return o, i * (eq + em + h.abs() * emh + eh * (mh.abs() + emh) + COST * U * (q.abs() + m.abs() + (h * mh).abs()))

    def total(v, e):
        return v.sum(0), (v.abs()).sum(0), e.sum(0)

    def finish(v, z, e):
        return _out(v, e + sr * z, dtype)

    got = {}
    t = _d(dout) if dout is not None else torch.zeros(R, d, dtype=torch.float64)
    et = torch.zeros_like(t)
    if dnormed is not None:
        dn = _d(dnormed)
        h, eh, i = normed(out, 2)
        q = dn if nw is None else dn * _d(nw)
        o, e = through(q, U * q.abs(), h, eh, i)
        et = e + 2 * U * (t.abs() + o.abs())
        t = t + o
        got["dnext_weight"] = finish(*total(dn * h, dn.abs() * eh))
        got["dnext_bias"] = finish(*total(dn, 0 * dn))
    if after:
        h, eh, i = normed(x, 0)
    else:
        h = _d(x) if x is not None else torch.zeros_like(t)
        eh = torch.zeros_like(h)
    g = _gate(gate, R, d)
    f = g if w is None else g * _d(w)
    q, eq = t * f, et * f.abs() + 3 * U * (t * f).abs()
    got["dx"] = _out(*(through(q, eq, h, eh, i) if after else (q, eq)), dtype)
    got["dresidual"] = _out(scale * t, abs(scale) * et + 2 * U * (scale * t).abs(), dtype)
    A = t * h
    eA = et * (h.abs() + eh) + t.abs() * eh
    if after:
        got["dweight"] = finish(*total(A * g, eA * g.abs()))
        got["dbias"] = finish(*total(t * g, et * g.abs()))
    if gate is not None:
        gates = 1 if gate.dim() == 1 else gate.shape[0]
        wv = torch.ones(d, dtype=torch.float64) if w is None or not after else _d(w)
        bv = torch.zeros(d, dtype=torch.float64) if b is None or not after else _d(b)
        per = lambda v: v.reshape(gates, -1, d).sum(1)  # noqa: E731
        v, z, e = per(A) * wv + per(t) * bv, per(A.abs()) * wv.abs() + per(t.abs()) * bv.abs(), \
            per(eA) * wv.abs() + per(et) * bv.abs()
        got["dgate"] = tuple(r.reshape(gate.shape) for r in finish(v, z, e))
    return got
