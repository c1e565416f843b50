"""The kernels of the 8-bit operators and the block norm themselves, run on the CPU
(cpu_kernels/block_main.cpp): every read and write of device memory checked against
tensors of exactly their size with the elements between rows forbidden, results
against loops in 64 bits (integers and scales exactly)."""
import random

import pytest

from cpu_kernels import build_block as C

TYPES = ["fp32", "bf16", "fp16"]

# strides and offsets of the first element, in elements
RAGGED = [dict(), dict(pad_x=1, pad_w=3, pad_y=2, pad_res=5, pad_q=7, pad_n=1), dict(off_x=1, off_w=3, off_y=5, off_res=2, off_q=3),
          dict(pad=8), dict(pad=8, off=8), dict(pad=16, off=16)]


def _run(cases, name=None):
    """Every case right; name: what each case's first launch must name."""
    out = C.run(cases)
    assert len(out) == len(cases)
    bad = ["%s: %s" % (c, r) for c, (r, _) in zip(cases, out) if r.split()[:2] != ["ok", "0"]]
    assert not bad, "\n".join(bad[:10])
    if name is not None:
        for c, (_, lines) in zip(cases, out):
            assert name in lines[0], (c, lines)
    return out


WIDTHS = ((1, 1), (3, 2), (5, 7), (300, 8), (9, 77), (33, 130), (40, 256), (9, 300), (17, 1000), (6, 2049), (5, 4096), (3, 5000),
          (2, 8192), (2, 8193), (3, 12001), (2, 17000), (0, 5), (700, 64), (41, 128))


@pytest.mark.parametrize("t", TYPES)
def test_quantize(t):
    cases = []
    for i, (R, d) in enumerate(WIDTHS):
        for j, r in enumerate(RAGGED):
            for group in (0, 128):
                cases.append(dict(op="quantize", type=t, rows=R, d=d, group=group, seed=i, special=(i + j) % 4, cus=(256, 1)[j % 2], **r))
                cases.append(dict(op="dequantize", type=t, rows=R, d=d, group=group, seed=i, **r))
    # values so small that the scale is the smallest one, and as large as the type has
    small, large = {"fp32": (1e-40, 1.9e38), "bf16": (1e-40, 1.9e38), "fp16": (1e-7, 38000.)}[t]
    cases += [dict(op="quantize", type=t, rows=9, d=d, group=128, size=s) for d in (5, 300) for s in (small, 1e-37, large)]
    _run(cases)


def _int8(t, size, i, **kw):
    M, K, N = size
    return dict(op="int8", type=t, M=M, K=K, N=N, act=i % 4, bias=int(i % 3 > 0), residual=int(i % 5 > 1), in_place=int(i % 7 == 3),
                seed=100 + i, **kw)


SIZES = ((1, 1, 1), (1, 15, 7), (1, 16, 8), (2, 64, 40), (3, 65, 39), (16, 1000, 17), (17, 129, 65), (31, 200, 9), (33, 96, 47),
         (64, 700, 130), (65, 7, 5), (128, 16, 128), (129, 130, 127), (200, 256, 264), (257, 400, 96), (130, 1040, 61), (300, 17, 9))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("cus", [1, 256])
def test_int8_products(t, cus):
    cases = []
    for i, size in enumerate(SIZES):
        for j, r in enumerate(RAGGED):
            cases.append(_int8(t, size, i + j, cus=cus, late=j % 2, **r))
    # the largest sums
    cases += [_int8(t, (3, K, 5), 1, cus=cus, most=1) for K in (131071, 131056)]
    _run(cases)


@pytest.mark.parametrize("t", TYPES)
def test_gradient_from_8_bits(t):
    cases = []
    for i, (M, K, N) in enumerate(((1, 1, 1), (1, 64, 72), (3, 7, 5), (40, 33, 24), (65, 1, 130), (130, 72, 136), (300, 140, 1),
                                   (1000, 24, 16), (0, 9, 5), (70, 260, 300))):
        for j, r in enumerate(RAGGED):
            for oi in (0, 1):
                cases.append(dict(op="backward_int8", type=t, M=M, K=K, N=N, oi=oi, act=(i + j) % 4, p=(0, 0.4, 1)[(i + j) % 3],
                                  x_group=128 * ((i + oi) % 2), pre_group=128 * (j % 2), want=7 if j < 2 else 1 + (i + j) % 7,
                                  pad_dy=j, pad_dx=2 * j, pad_dw=3 * j, pad_pre=j, seed=i, **r))
    _run(cases)


def _norm(op, t, R, d, i, j, **kw):
    gates = (0, 1, 1, 2, 3, R)[(i + j) % 6]
    if gates and R % gates:
        gates = 1
    after, before = ((1, 1), (1, 1), (1, 0), (0, 1))[(i + 2 * j) % 4]
    return dict(op=op, type=t, rows=R, d=d, gates=gates, after=after, before=before, rms=(i + j) % 2, scale=(1, 0.5, -2, 0)[j % 4],
                w=int((i + j) % 3 > 0), b=j % 2, seed=i, cus=(256, 1, 2)[j % 3], **kw)


NORM_WIDTHS = ((1, 1), (4, 2), (6, 7), (300, 8), (9, 77), (36, 130), (40, 256), (9, 300), (18, 1000), (6, 2049), (6, 4096), (3, 5000),
               (2, 8192), (2, 8193), (3, 12001), (2, 17000), (0, 5), (600, 64))


@pytest.mark.parametrize("t", TYPES)
def test_block_norm(t):
    cases = []
    for i, (R, d) in enumerate(NORM_WIDTHS):
        for j, r in enumerate(RAGGED):
            cases.append(_norm("block_norm", t, R, d, i, j, alias=(0, 1, 2, 3, 4, 0)[j], no_stats=int(j == 5), **r))
    _run(cases)


@pytest.mark.parametrize("t", TYPES)
def test_block_norm_gradient(t):
    cases = []
    for i, (R, d) in enumerate(NORM_WIDTHS):
        for j, r in enumerate(RAGGED):
            cases.append(_norm("block_norm_backward", t, R, d, i, j, alias=(0, 0, 1, 2, 0, 1)[j], no_dout=int(j == 4),
                               no_params=int(j == 3), pad_dy=j, pad_dn=j, **r))
    _run(cases)


@pytest.mark.parametrize("t", TYPES)
def test_block_norm_gradient_with_a_gate_for_every_row(t):
    cases = []
    for i, (R, d) in enumerate(NORM_WIDTHS[1:]):
        for j, r in enumerate(RAGGED):
            for after, before in ((1, 1), (1, 0), (0, 1)):
                c = _norm("block_norm_backward", t, R, d, i, j, alias=(0, 0, 1, 2, 0, 1)[j], no_dout=int(j == 4 and before),
                          no_params=int(j == 3), pad_dy=j, pad_dn=j, **r)
                cases.append(dict(c, gates=max(R, 1), after=after, before=before))
    if t != "fp16":  # (which has no 2^60)
        cases += [dict(op="block_norm_backward", type=t, rows=3, d=d, constant=2.0 ** 60, w=1, gates=3) for d in (1, 5, 130, 1025, 8191)]
    _run(cases)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_block_norm_gradient_of_large_constant_rows(t):
    # x - mean is zero in every column, though mean times rstd (eps^-0.5 = 316) is no
    # float: columns past the row's end, which fill its last pieces, add nothing
    _run([dict(op="block_norm_backward", type=t, rows=3, d=d, constant=2.0 ** 123, w=1, gates=1) for d in (1, 5, 16, 130, 300, 1025, 9000)])


def test_rows_far_apart():
    # offsets past 32 bits
    far = dict(ld_x=1 << 25, ld_y=1 << 25, ld_dy=1 << 25, ld_dx=1 << 25, ld_dr=1 << 25, ld_dn=1 << 25, ld_n=1 << 25, ld_res=1 << 25)
    _run([dict(op=op, type=t, rows=70, d=77, w=1, gates=1, group=128, **far)
          for t in TYPES for op in ("block_norm", "block_norm_backward")])
    far = {k: 1 << 26 for k in ("ld_x", "ld_w", "ld_q", "ld_pre")}
    _run([dict(op=op, type=t, rows=70, d=77, group=128, **far) for t in TYPES for op in ("quantize", "dequantize")])
    _run([_int8(t, (200, 130, 135), i, cus=1, ld_y=1 << 25, **far) for t in TYPES for i in (0, 1)])
    _run([_int8("bf16", (70, 144, 130), 1, ld_y=1 << 25, ld_x=1 << 26, ld_w=1 << 25)])
    _run([dict(op="backward_int8", type=t, M=70, K=40, N=33, act=2, x_group=128, ld_x=1 << 26, ld_pre=1 << 26) for t in TYPES])


def _draw(r):
    def log(a, b):
        return int(round(a * (b / a) ** r.random()))
    op = r.choice(["quantize", "dequantize", "int8", "int8", "int8", "backward_int8", "block_norm", "block_norm_backward"])
    c = dict(op=op, type=r.choice(TYPES), seed=r.randint(1, 10 ** 6), cus=r.choice([1, 2, 8, 64, 256]), p=r.choice([0, 0.3, 1]),
             late=r.randint(0, 1), group=r.choice([0, 128]))
    for n in ("x", "w", "y", "q", "n", "pre", "res", "dy", "dn", "dx", "dr", "dw"):
        if r.random() < 0.4:
            c["pad_" + n] = r.choice([1, 2, 3, 8, 16, r.randint(1, 40)])
        if r.random() < 0.25:
            c["off_" + n] = r.choice([1, 2, 4, 8, 16])
    if op in ("int8", "backward_int8"):
        M, K, N = log(1, 500), log(1, 1500), log(1, 500)
        if r.random() < 0.5:
            M, K, N = (M + 7) // 8 * 8, (K + 15) // 16 * 16, (N + 7) // 8 * 8
        while M * K * N > 2e7:
            M, K, N = M // 2 + 1, max(1, K // 32 * 16), N // 2 + 1
        return dict(c, M=M, K=K, N=N, oi=r.randint(0, 1), act=r.randint(0, 3), bias=r.randint(0, 1), residual=r.randint(0, 1),
                    in_place=int(r.random() < 0.2), want=r.randint(1, 7), x_group=r.choice([0, 128]), pre_group=r.choice([0, 128]))
    d = log(1, 20000)
    rows = log(1, max(2, 50000 // d))
    gates = r.choice([0, 1, r.randint(1, rows)])
    rows = rows // gates * gates if gates else rows
    after, before = r.choice([(1, 1), (1, 1), (1, 0), (0, 1)])
    return dict(c, rows=rows, d=d, gates=gates, after=after, before=before, rms=r.randint(0, 1), scale=r.choice([1, 0.5]),
                w=r.randint(0, 1), b=r.randint(0, 1), no_dout=int(r.random() < 0.2), alias=r.choice([0, 0, 1, 2]))


@pytest.mark.parametrize("seed", range(4))
def test_drawn_calls(seed):
    r = random.Random(seed)
    _run([_draw(r) for _ in range(60)])


def test_widest_calls():
    # nothing runs: every size that the header allows makes launches that HIP takes
    # (fewer than 2^32 threads along an axis), or is refused as one that it does not
    sizes = (1, 3, 8, 65, 1000, 16384, 1 << 24, (1 << 27) + 8, 1 << 30, (1 << 31) - 1)
    cases = []
    for t in ("fp32", "bf16"):
        for M in sizes:
            for d in sizes:
                if M * d < 1 << 40:
                    cases += [dict(op=op, type=t, rows=M, d=d, gates=g, group=128 * (M % 2), dry=1)
                              for op in ("quantize", "dequantize", "block_norm", "block_norm_backward") for g in (1, M)]
            for K in sizes:
                for N in sizes:
                    if max(M * K, M * N, K * N) < 1 << 40:
                        if K < 131072:
                            cases.append(dict(op="int8", type=t, M=M, K=K, N=N, dry=1))
                        cases.append(dict(op="backward_int8", type=t, M=M, K=K, N=N, act=3, dry=1))
    for c, (r, _) in zip(cases, C.run(cases)):
        size = c["M"] * max(c["K"], c["N"]) if "M" in c else c["rows"] * c["d"]
        assert r.split()[1] == "0" or (r.split()[1] == "5" and size > 1 << 35), (c, r)
        assert int(r.split()[2]) < 1 << 32, (c, r)


def test_which_kernel_an_int8_product_takes():
    def taken(name, cases):
        for c, (_, lines) in zip(cases, _run(cases)):
            assert name in lines[0], (c, lines)
        return cases
    for i, t in enumerate(TYPES):
        taken("few rows", [_int8(t, s, i, **r) for s in ((1, 4096, 40), (16, 1000, 17), (33, 520, 47), (64, 300, 33))
                           for r in (dict(), dict(pad=3), dict(off=5))])
        for kind, sizes, strides in (
                ("staged", ((65, 7, 5), (200, 130, 135), (130, 300, 260), (129, 1000, 64)), (dict(), dict(pad=3), dict(pad=16, off=1))),
                ("direct", ((65, 16, 8), (130, 144, 136), (257, 400, 96), (520, 592, 512), (264, 656, 520)),
                 (dict(), dict(pad_x=32, off=16, pad_y=1)))):
            out = _run([_int8(t, s, i, late=(i + j) % 2, cus=cus, **r) for s in sizes for r in strides for j, cus in enumerate((1, 8, 256))])
            tiles = {lines[0].split(", ")[1] for _, lines in out}
            assert tiles == {"%s tiles of %d" % (kind, n) for n in (64, 128, 256)[:2 if kind == "staged" else 3]}, tiles
        taken("panels", [dict(_int8(t, s, i + j, **r), cus=8)
                         for j, (s, r) in enumerate((((16384, 16, 128), dict()), ((16417, 37, 129), dict(pad=3)), ((2079, 64, 1030), dict(off=1)),
                                                     ((2049, 100, 1100), dict(pad=1)), ((8262, 128, 300), dict(pad=16))))])
        # a contraction in parts, joined
        for s in ((70, 2064, 72), (130, 4112, 61), (96, 3001, 130)):
            for _, lines in _run([_int8(t, s, i + j) for j in range(2)]):
                assert "tiles" in lines[0] and int(lines[0].rsplit(" ", 2)[1]) > 1, lines
