"""The 8-bit operators and the block norm on the GPU where their kernels' loops run long
and their choices meet: scales of both signs."""
import pytest
import torch

import block_oracle as B
import ff_oracle as O
import paper_2507_01040_amd as P
from test_feed_forward_gpu import DTYPES, ids
from test_residual_block_gpu import Eight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_dense_int8_scales_of_both_signs(dtype):
    # scales far from one whose product is an ordinary float, of either sign: few rows, tiles,
    # a split contraction, panels
    for M, K, N in ((3, 20000, 40), (70, 20016, 72), (300, 130, 65), (2100, 112, 1030)):
        v = Eight(61, dtype)
        x, w = torch.full((M, K), 127, dtype=torch.int8, device="cuda:0"), torch.full((N, K), -127, dtype=torch.int8, device="cuda:0")
        w[::3] = v.int8(w[::3].shape[0], K)
        xs, ws = v.scale(M), v.scale(N, size=1 / (16000 * K))
        xs[1::2] *= -1
        ws[::4] *= -1
        for far in (118, -118):
            a, b = torch.ldexp(xs, torch.tensor(far)), torch.ldexp(ws, torch.tensor(-far))
            y = P.dense_int8(x, a, w.t(), b, dtype=dtype)
            O.check(y, B.dense_int8(x, a, w.t(), b, None, 0, None, dtype), "y of %s" % ((M, K, N, far),))
