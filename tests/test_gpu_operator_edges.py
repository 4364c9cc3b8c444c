"""The operators on loaded weights at the edges of their formats, types and sizes.

Tolerances are those of ``test_gpu_operators``: a sum of `depth` products in 32
bits is off by at most `sum_bound`, and an output's rounding adds half a unit in
its last place.
"""

import numpy as np
import pytest

from oracle import operators_oracle as O
from tests.test_gpu_operators import TYPES, assert_close, host, normal, random_mx4, sum_bound

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import operators as op  # noqa: E402


@pytest.fixture(autouse=True)
def _device(gpu_device):
    return gpu_device


def values(w):
    return O.dequantize(w.codes.cpu().numpy(), w.scales.cpu().numpy(), w.cols)


# rows on both sides of the kernel of few rows, and tiles of every height
ROWS = [(1, 200, 320), (5, 200, 320), (16, 200, 320), (17, 200, 320), (40, 200, 320), (130, 200, 320), (300, 2100, 320),
        (3300, 3600, 96), (3300, 96, 3600)]


# ---- blocks and elements that float16 does not hold -------------------------

@pytest.mark.parametrize("m,n,k", ROWS)
@pytest.mark.parametrize("scale", [0, 96, 133, 246, 247, 254])
def test_block_of_zeros_under_any_scale(m, n, k, scale):
    """A block of zeros, of either sign, stands for zeros whatever its scale."""
    w, _ = random_mx4(n, k, m + scale, (116, 128))
    for row, block, code in ((7, 1, 0x00), (n - 1, (k - 1) // 32, 0x88), (n // 2, 0, 0x08)):
        w.codes[row, block * 16:(block + 1) * 16] = code
        w.scales[row, block] = scale
    wv = values(w)
    for dtype in TYPES:
        x, dy = normal((m, k), dtype, 1), normal((m, n), dtype, 2)
        a, b = host(x), host(dy)
        assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, k), torch.float32)
        assert_close(op.mx4_linear_grad(dy, w, out_dtype=torch.float32), O.linear_grad(b, wv), sum_bound(b, wv, n), torch.float32)
