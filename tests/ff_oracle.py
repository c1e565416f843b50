"""Plain implementations in 64 bits of the feed-forward operators (layer norm,
dense layer, dropout, their gradients), on the CPU, and the error bounds of
their tests.

Bounds.  u is the unit roundoff of a type (2^-24, 2^-8, 2^-11), U that of the
32-bit sums.  A sum of n rounded terms t_i in any order differs from the exact
one by at most about sqrt(n) U sum |t_i| times a small constant (rounding errors
of independent signs; Higham and Mary, SIAM J. Sci. Comput. 41, 2019); LAMBDA =
8 standard deviations are allowed.  Everything that follows a sum adds a few
U of its operands (COST of them are allowed), and the output one u.  Smallest
floats add an absolute term.
"""
import numpy as np
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}
LAMBDA, COST = 8.0, 16.0
SLOPE = 1.13  # largest slope of the activations


def philox_words(key, step, rows, cols, first_row=0):
    """Words of Philox4x32-7 for a rows x cols matrix, uint32."""
    q = np.arange((cols + 3) // 4, dtype=np.uint64)
    r = np.arange(first_row, first_row + rows, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    c = [np.broadcast_to(q, (rows, q.size)), np.broadcast_to((r & m)[:, None], (rows, q.size)),
         np.broadcast_to((r >> np.uint64(32))[:, None], (rows, q.size)),
         np.full((rows, q.size), step & 0xFFFFFFFF, np.uint64)]
    k0, k1 = key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF
    for _ in range(7):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, -1).reshape(rows, -1)[:, :cols].astype(np.uint32)


def mask(dropout, rows, cols):
    """1 / (1 - p) where kept, 0 where dropped (float64), or None."""
    if dropout is None:
        return None
    p, (key, step) = dropout
    if p == 1.0:
        return torch.zeros(rows, cols, dtype=torch.float64)
    keep = philox_words(key, step, rows, cols).astype(np.uint64) >= round(p * 2.0 ** 32)
    return torch.from_numpy(keep.astype(np.float64) / (1.0 - p))


def _times(v, m):
    # dropped elements are zero whatever they were
    return v if m is None else torch.where(m == 0, torch.zeros_like(v), v * m)


def _phi(v):
    # torch's ndtr loses the left tail to cancellation (1e-16 of 1)
    return 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)


def act(a, v):
    if a == 1:
        return torch.clamp(v, min=0.0)
    if a == 2:
        return v * _phi(v)
    if a == 3:
        return v * torch.sigmoid(v)
    return v


def slope(a, v):
    if a == 1:
        return (v > 0).double()
    if a == 2:
        return _phi(v) + v * torch.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    if a == 3:
        s = torch.sigmoid(v)
        return s + v * s * (1 - s)
    return torch.ones_like(v)


def _d(t):
    return None if t is None else t.detach().cpu().double()


def dense(x, w, b, a, dropout, res, dtype):
    """((y, bound), (pre, bound))."""
    x, w, b, res = _d(x), _d(w), _d(b), _d(res)
    K = x.shape[1]
    pre = x @ w
    size = x.abs() @ w.abs()
    if b is not None:
        pre, size = pre + b, size + b.abs()
    e = (LAMBDA * K ** 0.5 + COST) * U * size
    m = mask(dropout, *pre.shape)
    f = act(a, pre)
    y, ey = f, SLOPE * e + COST * U * (f.abs() + (pre.abs() if a else 0))
    y = _times(y, m)
    ey = _times(ey, m)
    if res is not None:
        y, ey = y + res, ey + 2 * U * res.abs()
    u, t = UNIT[dtype], TINY[dtype]
    return (y, ey * (1 + u) + 2 * u * y.abs() + t), (pre, e * (1 + u) + 2 * u * pre.abs() + t)


def dense_backward(dy, x, w, pre, a, dropout, dtype):
    """((dx, bound), (dw, bound), (db, bound))."""
    dy, x, w, pre = _d(dy), _d(x), _d(w), _d(pre)
    M, N = dy.shape
    K = x.shape[1]
    g = dy
    m = mask(dropout, M, N)
    eg = torch.zeros_like(g)
    if a:
        g = g * slope(a, pre)
        eg = COST * U * dy.abs() * (1 + pre.abs())
    g, eg = _times(g, m), _times(eg, m)
    u, t = UNIT[dtype], TINY[dtype]
    eg = eg + 2 * U * g.abs()
    # g is rounded once for the products
    er = eg + (u * g.abs() + t if a or m is not None else 0)

    def out(v, size, n, e):
        e = e + (LAMBDA * n ** 0.5 + COST) * U * size
        return v, e * (1 + u) + 2 * u * v.abs() + t

    ga = g.abs()
    return (out(g @ w.t(), ga @ w.abs().t(), N, er @ w.abs().t()),
            out(x.t() @ g, x.abs().t() @ ga, max(M, 1), x.abs().t() @ er),
            out(g.sum(0), ga.sum(0), max(M, 1), eg.sum(0)))


def layer_norm(x, w, b, eps, dtype):
    """((y, bound), (mean, bound), (rstd, bound))."""
    x, w, b = _d(x), _d(w), _d(b)
    d = x.shape[1]
    s = (LAMBDA * d ** 0.5 + COST) * U
    mean = x.mean(1)
    em = s * x.abs().mean(1)
    c = x - mean[:, None]
    var = (c * c).mean(1)
    rstd = (var + eps) ** -0.5
    # the variance about a mean that is em off: + em^2, and its own sum
    er = rstd * (0.5 * (em ** 2 + s * var + 2 * U * eps) * rstd ** 2 + 4 * U)
    h = c * rstd[:, None]
    eh = (em[:, None] + U * x.abs()) * rstd[:, None] + c.abs() * er[:, None] + 4 * U * h.abs()
    y, ey = h, eh
    if w is not None:
        y, ey = y * w, ey * w.abs() + 2 * U * (y * w).abs()
    if b is not None:
        ey = ey + 2 * U * (y.abs() + b.abs())
        y = y + b
    u, t = UNIT[dtype], TINY[dtype]
    return (y, ey * (1 + u) + 2 * u * y.abs() + t), (mean, em + t), (rstd, er + t)


def layer_norm_backward(dy, x, mean, rstd, w, res, dtype):
    """((dx, bound), (dw, bound), (db, bound)) for the given statistics."""
    dy, x, mean, rstd, w, res = (_d(v) for v in (dy, x, mean, rstd, w, res))
    R, d = x.shape
    s = (LAMBDA * d ** 0.5 + COST) * U
    i = rstd[:, None]
    h = (x - mean[:, None]) * i
    eh = 4 * U * (h.abs() + (x.abs() + mean.abs()[:, None]) * i)
    q = dy if w is None else dy * w
    mq, mqh = q.mean(1, keepdim=True), (q * h).mean(1, keepdim=True)
    emq = s * q.abs().mean(1, keepdim=True)
    emqh = s * (q * h).abs().mean(1, keepdim=True) + (q.abs() * eh).mean(1, keepdim=True)
    dx = i * (q - mq - h * mqh)
    e = i * (emq + h.abs() * emqh + eh * mqh.abs() + COST * U * (q.abs() + mq.abs() + (h * mqh).abs()))
    if res is not None:
        e = e + 2 * U * (dx.abs() + res.abs())
        dx = dx + res
    u, t = UNIT[dtype], TINY[dtype]
    sr = (LAMBDA * max(R, 1) ** 0.5 + COST) * U

    def out(v, size, e):
        e = e + sr * size
        return v, e * (1 + u) + 2 * u * v.abs() + t

    return ((dx, e * (1 + u) + 2 * u * dx.abs() + t),
            out((dy * h).sum(0), (dy * h).abs().sum(0), (dy.abs() * eh).sum(0)),
            out(dy.sum(0), dy.abs().sum(0), torch.zeros(d, dtype=torch.float64)))


def dropout(x, drop, res, dtype):
    x, res = _d(x), _d(res)
    y = _times(x, mask(drop, *x.shape))
    e = 2 * U * y.abs()
    if res is not None:
        e = e + 2 * U * (y.abs() + res.abs())
        y = y + res
    u, t = UNIT[dtype], TINY[dtype]
    return y, e * (1 + u) + 2 * u * y.abs() + t


def check(got, want, what=""):
    """Every element of got within the bound of (value, bound)."""
    v, e = want
    g = got.detach().cpu().double()
    assert g.shape == v.shape, (what, g.shape, v.shape)
    fine = torch.isfinite(v)
    assert torch.equal(torch.isnan(g), torch.isnan(v)), "%s: NaN in other places" % what
    assert torch.equal(g[~fine & ~torch.isnan(v)], v[~fine & ~torch.isnan(v)]), "%s: infinities" % what
    off = ((g - v).abs() - e)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, "%s: %g over its bound (%d of %d elements)" % (
        what, float(off.max()), int((off > 0).sum()), off.numel())
