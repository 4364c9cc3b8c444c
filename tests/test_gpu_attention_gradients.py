"""Gradients of attention where scores are far from zero, and where rows end inside a tile, against the oracle's 64-bit
definitions; tolerances are those of test_gpu_attention."""

import math

import numpy as np
import pytest

from tests.test_gpu_attention import TYPES, check, host, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import operators as op  # noqa: E402


@pytest.fixture(autouse=True)
def _device(gpu_device):
    return gpu_device


def shifted(lengths, heads, kv, dim, dtype, shift):
    """q, k, v and dout with scores of about `shift`, by one element of q and k."""
    n = sum(lengths)
    q, k, v = (normal((n, h, dim), dtype, i, 0.3) for i, h in enumerate((heads, kv, kv)))
    q[..., 0] = 4.0
    k[..., 0] = shift * dim ** 0.5 / 4
    return q, k, v, normal((n, heads, dim), dtype, 3, 0.1)


# Sinks, and texts longer than the window: the rows that see a tile of keys are no multiple of 32, in the window
# and behind it; by one workgroup and by several.  The fourth has sinks in more than one tile, the fifth rows behind
# the window in two parts, the last several texts of which some have none.
ENDS = [([901], 3, 1, 64, 1, 1), ([701, 450], 5, 1, 80, 300, 4), ([1000], 2, 2, 128, 37, 2), ([700], 3, 3, 33, 20, 130),
        ([899], 6, 2, 40, 129, 3), ([301, 5, 0, 170, 477], 3, 3, 64, 40, 2)]


@pytest.mark.parametrize("shift", [-1.0, -3.0, -20.0, -100.0])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(ENDS)))
def test_rows_past_the_end_weigh_nothing(case, dtype, shift):
    lengths, heads, kv, dim, window, sinks = ENDS[case]
    q, k, v, dout = shifted(lengths, heads, kv, dim, dtype, shift)
    check(q, k, v, lengths, window, sinks, dtype, dout=dout)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_sink_of_minus_infinity(dtype):
    """A key that no one can weigh: its gradients are zeros, and rows past the end make nothing else of them."""
    q, k, v, dout = shifted([901], 3, 1, 64, dtype, -3.0)
    q[..., 1] = q[..., 1].abs() + 1
    k[1, :, 1] = -math.inf
    leaves = [t.requires_grad_() for t in (q, k, v)]
    _, dk, dv = torch.autograd.grad(op.attention(*leaves, window=40, sinks=3), leaves, dout)
    assert not dk[1].any() and not dv[1].any()
    assert torch.isfinite(dk).all() and torch.isfinite(dv).all()
