"""The feed-forward kernels themselves, run on the CPU (cpu_kernels/main.cpp): every
read and write of device memory checked against tensors of exactly their size with
the elements between rows forbidden, results against loops in 64 bits, and which
kernel a call takes."""
import random

import pytest

from cpu_kernels import build as C
from ff_cases import LARGE_TILES

TYPES = ["fp32", "bf16", "fp16"]


def _run(cases, kernels=None):
    """Every case right; kernels: what each case's launches must name, in order."""
    out = C.run(cases)
    assert len(out) == len(cases)
    bad = ["%s: %s" % (c, r) for c, (r, _) in zip(cases, out) if r.split()[:2] != ["ok", "0"]]
    assert not bad, "\n".join(bad[:10])
    if kernels is not None:
        for c, (_, lines) in zip(cases, out):
            lines = [s for s in lines if s.startswith("cliffconv: product")]
            assert len(lines) == len(kernels) and all(k in s for k, s in zip(kernels, lines)), (c, lines)
    return out


def _dense(t, size, i, **kw):
    """A dense layer of that size; i varies order, epilogue, strides and alignment."""
    M, K, N = size
    c = dict(op="dense", type=t, M=M, K=K, N=N, oi=i & 1, act=i % 4, bias=i % 3 > 0, residual=i % 5 > 1, pre=i % 2,
             p=(0, 0.3, 0, 1)[i % 4 if i % 3 else 0], in_place=i % 7 == 3, seed=100 + i)
    c.update({k: int(v) for k, v in c.items() if isinstance(v, bool)})
    c.update(kw)
    return c


# strides and offsets of the first element, in elements
RAGGED = [dict(), dict(pad_x=1, pad_w=3, pad_y=2, pad_res=5, pad_pre=1), dict(off_x=1, off_w=3, off_y=5, off_res=2),
          dict(pad=8), dict(pad=8, off=8)]


@pytest.mark.parametrize("t", TYPES)
def test_few_rows(t):
    cases = []
    for size in ((1, 8, 8), (1, 64, 64), (1, 72, 33), (2, 520, 40), (3, 65, 39), (16, 1000, 17), (17, 129, 65), (31, 200, 9),
                 (33, 96, 47), (64, 700, 130), (50, 63, 31)):
        for i, r in enumerate(RAGGED):
            cases += [_dense(t, size, i, **r), _dense(t, size, i + 5, **r)]
    _run(cases, ["few rows"])


@pytest.mark.parametrize("t,name", [("fp32", "split tiles of 128"), ("bf16", "staged tiles of 128"),
                                    ("fp16", "staged tiles of 128")])
def test_tiles(t, name):
    # (one compute unit: the contraction is not split); widths that are not whole pieces
    cases = []
    for size in ((65, 7, 5), (70, 1, 1), (128, 3, 130), (129, 65, 127), (200, 130, 135), (300, 17, 9), (131, 203, 258)):
        for i, r in enumerate(RAGGED):
            cases += [_dense(t, size, i, cus=1, **r), _dense(t, size, i + 5, cus=1, **r)]
    _run(cases, [name + ", "])


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_direct_tiles(t):
    aligned = [dict(), dict(pad=8), dict(pad_x=16, pad_w=8, pad_y=1, off_y=1, pad_res=3)]
    small = [(65, 8, 8), (130, 72, 136), (128, 64, 128), (200, 136, 264), (257, 200, 96)]
    _run([_dense(t, s, i + 3 * j, late=j, **r) for s in small for i, r in enumerate(aligned) for j in range(2)],
         ["direct tiles of 128, "])
    # 256 x 256: ragged edges, a last stage that is not whole, one and two stages
    large = [(520, 1096, 512), (513, 840, 488), (1000, 600, 264), (264, 648, 1000), (257, 1048, 512)]
    _run([_dense(t, s, i + 3 * j, cus=1, late=j, **r) for s in large for i, r in enumerate(aligned[:2]) for j in range(2)],
         ["direct tiles of 256, "])


@pytest.mark.parametrize("t", TYPES)
def test_split_contraction(t):
    cases = [_dense(t, size, i, **r) for i, size in enumerate(((70, 1000, 72), (130, 2056, 61), (96, 1531, 250), (100, 1024, 8)))
             for r in RAGGED]
    for _, lines in _run(cases):
        assert "tiles" in lines[0] and int(lines[0].rsplit(" ", 2)[1]) > 1, lines
    # outputs enough for the join of one thread per group
    _run([_dense(t, (1003, 200, 777), 2, cus=4096)])


@pytest.mark.parametrize("t", TYPES)
def test_panels(t):
    cases = [_dense(t, (16384 + m, k, n), i, cus=8, **RAGGED[i % 5])
             for i, (m, k, n) in enumerate(((0, 8, 8), (33, 13, 5), (1, 64, 129), (70, 100, 40), (31, 128, 72), (5, 77, 1)))]
    _run(cases, ["panels"])


@pytest.mark.parametrize("t", TYPES)
def test_gradient(t):
    cases = []
    for i, (M, K, N) in enumerate(((1, 1, 1), (1, 64, 72), (3, 7, 5), (40, 33, 24), (65, 1, 130), (130, 72, 136), (300, 40, 1),
                                   (1000, 24, 16), (0, 9, 5), (16400, 16, 24), (16390, 9, 130))):
        for j, r in enumerate(RAGGED if M < 1000 else RAGGED[i % 2:i % 2 + 1]):
            for oi in (0, 1) if M < 1000 else (i % 2,):
                cases.append(dict(op="backward", type=t, M=M, K=K, N=N, oi=oi, act=(i + j) % 4, p=(0, 0.4, 1)[(i + j) % 3],
                                  want=7 if j < 2 else 1 + (i + j) % 7, pad_dy=j, pad_dx=2 * j, pad_dw=3 * j, seed=i, **r))
    _run(cases)


@pytest.mark.parametrize("t", TYPES)
def test_norm_and_dropout(t):
    cases = []
    for i, (R, d) in enumerate(((1, 1), (3, 2), (5, 7), (300, 8), (9, 77), (33, 130), (40, 256), (9, 300), (17, 1000), (6, 2049),
                                (5, 4096), (3, 5000), (2, 8192), (2, 8193), (3, 12001), (2, 17000), (0, 5), (700, 64))):
        for j, r in enumerate(RAGGED):
            flags = dict(w=(i + j) % 3 > 0, b=j % 2, residual=(i + j) % 2, in_place=j == 4, no_stats=j == 3)
            flags = {k: int(v) for k, v in flags.items()}
            cases.append(dict(op="norm", type=t, rows=R, d=d, seed=i, cus=(256, 1, 2)[j % 3], **flags, **r))
            cases.append(dict(op="norm_backward", type=t, rows=R, d=d, seed=i, cus=(256, 1, 2)[j % 3],
                              want=(6, 6, 0, 2, 4)[j], **flags, **r))
            cases.append(dict(op="dropout", type=t, rows=R, d=d, seed=i, p=(0, 0.3, 0.5, 1, 0.9)[j], **flags, **r))
    _run(cases)


def test_rows_far_apart():
    # offsets past 32 bits: row strides at the limits of the kernels that have them
    far = dict(ld_x=1 << 23, ld_y=1 << 23, ld_res=1 << 23, ld_pre=1 << 23, residual=1, pre=1, bias=1)
    _run([_dense("fp32", (64, 72, 40), 0, **far), _dense("fp32", (33, 200, 24), 1, ld_w=1 << 23, **far),
          _dense("bf16", (64, 136, 40), 0, ld_w=1 << 23, **far), _dense("fp16", (40, 264, 33), 1, ld_w=1 << 23, **far)], ["few rows"])
    far = {k: (1 << 21 if k[:2] == "ld" else v) for k, v in far.items()}
    _run([_dense("bf16", (300, 136, 136), i, ld_w=1 << 21, **far) for i in (0, 1)], ["direct tiles of 128, "])
    _run([_dense("bf16", (520, 1096, 512), i, cus=1, ld_w=1 << 21, **far) for i in (0, 1)], ["direct tiles of 256, "])
    far = dict(ld_x=(1 << 25) + 1, ld_y=(1 << 25) + 1, ld_res=(1 << 25) + 3, ld_w=(1 << 24) + 1, residual=1)
    _run([_dense(t, (200, 130, 135), i, cus=1, **far) for t in TYPES for i in (0, 1)])
    _run([dict(op=op, type=t, rows=70, d=77, ld_x=1 << 25, ld_y=1 << 25, ld_dy=1 << 25, ld_dx=1 << 25, w=1, p=0.5)
          for t in TYPES for op in ("norm", "norm_backward", "dropout")])


def _draw(r):
    def log(a, b):
        return int(round(a * (b / a) ** r.random()))
    op = r.choice(["dense", "dense", "backward", "backward", "norm", "norm_backward", "dropout"])
    c = dict(op=op, type=r.choice(TYPES), seed=r.randint(1, 10 ** 6), cus=r.choice([1, 2, 8, 64, 256]), p=r.choice([0, 0.3, 1]),
             late=r.randint(0, 1),
             in_place=int(r.random() < 0.2), residual=r.randint(0, 1))
    for n in ("x", "w", "y", "pre", "res", "dy", "dx", "dw"):
        if r.random() < 0.4:
            c["pad_" + n] = r.choice([1, 2, 3, 8, 16, r.randint(1, 40)])
        if r.random() < 0.25:
            c["off_" + n] = r.choice([1, 2, 4, 8])
    if op in ("dense", "backward"):
        M, K, N = log(1, 500), log(1, 700), log(1, 500)
        if r.random() < 0.5:
            M, K, N = (M + 7) // 8 * 8, (K + 7) // 8 * 8, (N + 7) // 8 * 8
        while M * K * N > 2e7:
            M, K, N = M // 2 + 1, K // 2 + 1, N // 2 + 1
        return dict(c, M=M, K=K, N=N, oi=r.randint(0, 1), act=r.randint(0, 3), bias=r.randint(0, 1), pre=r.randint(0, 1),
                    want=r.randint(1, 7))
    d = log(1, 20000)
    return dict(c, rows=log(1, max(2, 50000 // d)), d=d, w=r.randint(0, 1), b=r.randint(0, 1), want=r.choice([0, 2, 4, 6]))


@pytest.mark.parametrize("seed", range(4))
def test_drawn_calls(seed):
    r = random.Random(seed)
    _run([_draw(r) for _ in range(60)])


def test_widest_calls():
    # nothing runs: every size that the header allows makes launches that HIP takes
    # (fewer than 2^32 threads along an axis)
    sizes = (1, 3, 8, 65, 1000, 16384, 1 << 24, (1 << 27) + 8, 1 << 30, (1 << 31) - 1)
    cases = []
    for t in ("fp32", "bf16"):
        for M in sizes:
            for K in sizes:
                for N in sizes:
                    if max(M * K, M * N, K * N) < 1 << 40:
                        for oi in (0, 1):
                            cases.append(dict(op="dense", type=t, M=M, K=K, N=N, oi=oi, dry=1))
                            cases.append(dict(op="backward", type=t, M=M, K=K, N=N, oi=oi, act=3, dry=1))
            for d in sizes:
                if M * d < 1 << 40:
                    cases += [dict(op=op, type=t, rows=M, d=d, p=0.5, dry=1) for op in ("norm", "norm_backward", "dropout")]
    for r, _ in _run(cases):
        assert 0 < int(r.split()[2]) < 1 << 32


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_norm_gradient_of_large_constant_rows(t):
    # x - mean is zero in every column, though mean times rstd (eps^-0.5 = 316) is no
    # float: columns past the row's end, which fill its last pieces, add nothing
    _run([dict(op="norm_backward", type=t, rows=3, d=d, constant=2.0 ** 123, w=1, residual=1)
          for d in (1, 5, 16, 130, 300, 1025, 9000)])


def test_large_tiles_of_the_gpu_tests():
    # which kernels the calls of test_feed_forward_edges_gpu.py take
    for (M, K, N), forward, backward in LARGE_TILES:
        for t in ("bf16", "fp16"):
            for oi in (0, 1):
                _run([dict(op="dense", type=t, M=M, K=K, N=N, oi=oi, dry=1)], forward)
                if backward:
                    _run([dict(op="backward", type=t, M=M, K=K, N=N, oi=oi, dry=1)],
                         backward)
