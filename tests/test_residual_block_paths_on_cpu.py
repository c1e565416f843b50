"""The kernels of the 8-bit operators and the block norm on the CPU (cpu_kernels/
block_main.cpp, every access checked) where their loops run long and their choices meet."""
import itertools

import pytest

from block_cases import STEADY, stages
from cpu_kernels import build_block as C
from test_residual_block_on_cpu import RAGGED, TYPES, _run


def _weight_line(lines):
    return next(s for s in lines if "8-bit tiles" in s)


@pytest.mark.parametrize("t", TYPES)
def test_steady_loop_of_the_weight_gradient(t):
    # whole stages from five on, odd and even, with and without rows left; tiles at the edges beside them
    cases = [dict(op="backward_int8", type=t, M=M, K=K, N=N, oi=oi, act=2 + (i + j) % 2, p=(0, 0.4)[i % 2], x_group=128 * (j % 2),
                  pre_group=128 * (i % 2), want=2 + 4 * (i % 2), seed=i, cus=1, late=j % 2, **r)
             for i, (M, K, N) in enumerate(((160, 128, 128), (165, 128, 256), (192, 128, 128), (229, 256, 128), (288, 128, 128), (300, 140, 260)))
             for j, r in enumerate(RAGGED[:4]) for oi in (0, 1)]
    if t == "fp32":
        cases += [dict(cases[0], act=a, M=M) for a in (0, 1) for M in (197, 256)]
    for c, (_, lines) in zip(cases, _run(cases)):
        assert stages(c["M"], _weight_line(lines)) >= 5, (c, lines)


def test_steady_sizes_of_the_gpu_tests():
    for (M, K, N), line in STEADY:
        assert stages(M, line) >= 5
        for t, oi in itertools.product(TYPES, (0, 1)):
            (_, lines), = C.run([dict(op="backward_int8", type=t, M=M, K=K, N=N, oi=oi, act=2, dry=1)])
            assert line in _weight_line(lines), lines


@pytest.mark.parametrize("t", TYPES)
def test_products_with_scales_of_both_signs(t):
    # far from one, with a product that is an ordinary float, and the largest sums
    _run([dict(op="int8", type=t, M=M, K=K, N=N, far=far, most=1, bias=0, act=0, cus=cus, seed=i)
          for i, (M, K, N) in enumerate(((3, 131071, 5), (70, 2064, 72), (130, 300, 65), (2100, 112, 1030)))
          for far in (118, -118) for cus in (1, 256)])


@pytest.mark.parametrize("t", TYPES)
def test_block_norm_of_every_choice(t):
    cases = []
    for R, d, gates in ((40, 96, (0, 1, 4, 20, 40)), (24, 300, (2, 12, 24)), (12, 2049, (1, 6)), (12, 5000, (0, 3)), (8, 8200, (0, 1, 4, 8))):
        for n, ((after, before), rms, g) in enumerate(itertools.product(((1, 1), (1, 0), (0, 1)), (0, 1), gates)):
            c = dict(type=t, rows=R, d=d, gates=g, after=after, before=before, rms=rms, scale=(0.5, -2)[n % 2], w=1, b=1, seed=n,
                     cus=(1, 256)[n % 2], **RAGGED[n % len(RAGGED)])
            cases += [dict(c, op="block_norm", alias=a) for a in (0, 1 + n % 4)]
            cases += [dict(c, op="block_norm_backward", alias=a, no_dout=int(n % 5 == 4 and before)) for a in (0, 1 + n % 2)]
    _run(cases)
