"""The kernels of the 8-bit operators and the block norm on the CPU (cpu_kernels/
block_main.cpp, every access checked) where their loops run long and their choices meet."""
import pytest

from test_residual_block_on_cpu import TYPES, _run


@pytest.mark.parametrize("t", TYPES)
def test_products_with_scales_of_both_signs(t):
    # far from one, with a product that is an ordinary float, and the largest sums
    _run([dict(op="int8", type=t, M=M, K=K, N=N, far=far, most=1, bias=0, act=0, cus=cus, seed=i)
          for i, (M, K, N) in enumerate(((3, 131071, 5), (70, 131056, 8), (70, 2064, 72), (130, 300, 65), (2100, 112, 1030)))
          for far in (118, -118) for cus in (1, 256)])
