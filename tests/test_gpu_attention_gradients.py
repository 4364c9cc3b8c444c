"""Gradients of attention where scores are far from zero, and where rows end inside a tile, against the oracle's 64-bit
definitions; tolerances are those of test_gpu_attention."""

import math

import numpy as np
import pytest

from oracle import layer_oracle as O
from tests.test_gpu_attention import FLUSH, TYPES, UNIT, assert_within, check, host, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import binding, operators as op  # noqa: E402


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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [8, 10, 17, 20, 24, 29])
@pytest.mark.parametrize("order", ["up", "down", "only", "below"])
@pytest.mark.parametrize("window,sinks", [(None, 0), (100, 3)])
def test_gradients_of_scores_far_from_zero(dtype, power, order, window, sinks):
    """Scores of a large power of two, either sign, and something small, which 32 bits hold exactly.

    A row's weights against its largest score then have exponents below 127 that are exact but for the product with
    log2 e (2^-24 of it, twice), and a sum that divides them whose logarithm is off by 2^-23 of at most 9: less than
    2^-15 of a weight.  Logarithms of rows' sums up to 2^9 go through 32 bits, with four roundings: less than 2^-13.  Beyond
    that the output, of which delta is made, is off by half a step of its weights and of itself, and weights are rounded
    to the type."""
    n, heads, kv, dim = 301, 3, 1, 64
    u, e = UNIT[dtype], 2.0 ** -24
    step = max(2.0 ** (power - 23), 2.0 ** -4)
    x = normal((n,), torch.float32, 5)
    x = (x / step).round() * step if power < 24 else torch.zeros_like(x)
    third = torch.arange(n, device="cuda") * 3 // n - 1.0  # -1, 0, 1
    sign = {"up": third, "down": -third, "only": torch.ones_like(third), "below": -torch.ones_like(third)}[order]
    q, k = torch.zeros(n, heads, dim, device="cuda"), torch.zeros(n, kv, dim, device="cuda")
    q[..., 0], q[..., 1] = 2.0 ** (power // 2), 1
    k[..., 0], k[..., 1] = (sign * 2.0 ** (power - power // 2))[:, None], x[:, None]
    q, k, v, dout = q.to(dtype), k.to(dtype), normal((n, kv, dim), dtype, 7), normal((n, heads, dim), dtype, 8, 0.01)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(op.attention(*leaves, window=window, sinks=sinks, scale=1.0), leaves, dout)

    Q, K, V, D = (host(t) for t in (q, k, v, dout))
    seen = O.visible(range(n), range(n), window, sinks)
    want = [[np.zeros(t.shape), np.zeros(t.shape)] for t in (Q, K, V)]
    w = 2.0 ** -13
    sums = 4 * (heads * n + 16) * e
    for h in range(heads):
        g = h * kv // heads
        out, p, _ = O.attend(Q[:, h], K[:, g], V[:, g], seen, 1.0)
        e_out = (u + w + sums) * (p @ np.abs(V[:, g])) + u * np.abs(out) + FLUSH
        dp, delta = D[:, h] @ V[:, g].T, (D[:, h] * out).sum(1, keepdims=True)
        ds = np.where(seen, p * (dp - delta), 0.0)
        e_dp = 2 * (dim + 8) * e * (np.abs(D[:, h]) @ np.abs(V[:, g]).T + (np.abs(D[:, h]) * np.abs(out)).sum(1, keepdims=True)) + \
            (np.abs(D[:, h]) * e_out).sum(1, keepdims=True)
        # (float16's ds are times a power of two that a row or key keeps: 2^-36 of the largest for the small)
        small = 2.0 ** -36 * (dtype == torch.float16)
        e_ds = np.where(seen, p * e_dp + np.abs(ds) * (u + w + 8 * e) + FLUSH, 0.0)
        e_q, e_k = e_ds + small * np.abs(ds).max(1, keepdims=True), e_ds + small * np.abs(ds).max(0, keepdims=True)
        for i, (value, bound) in enumerate(((ds @ K[:, g], e_q @ np.abs(K[:, g]) + sums * (np.abs(ds) @ np.abs(K[:, g]))),
                                            (ds.T @ Q[:, h], e_k.T @ np.abs(Q[:, h]) + sums * (np.abs(ds).T @ np.abs(Q[:, h]))),
                                            (p.T @ D[:, h], ((u + w + sums) * p).T @ np.abs(D[:, h]) +
                                             (FLUSH + 2.0 ** -40) * (seen.T @ np.abs(D[:, h]))))):
            to = h if i == 0 else g
            want[i][0][:, to] += value
            want[i][1][:, to] += bound
    for name, t, (value, bound) in zip(("dq", "dk", "dv"), got, want):
        assert_within(t, value, bound, dtype, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,kv,dim,window,sinks", [([150, 0, 70, 301], 6, 2, 33, None, 0), ([500], 8, 1, 128, 60, 2),
                                                               ([700, 3], 2, 2, 80, 20, 1), ([40] * 9, 40, 1, 16, 7, 3)])
def test_layouts_of_scores_far_from_zero(lengths, heads, kv, dim, window, sinks, dtype):
    """Scores of about 1500 that differ by tens, as those of ordinary size: within the bounds that these have by size."""
    q, k, v, dout = shifted(lengths, heads, kv, dim, dtype, 1500.0)
    check(q, k, v, lengths, window, sinks, dtype, dout=dout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(None, 0), (50, 2), (2, 0)])
def test_rows_beside_one_far_from_zero(dtype, window, sinks):
    """A row of large scores changes its own gradient and its keys', no other row's, by not one bit.

    By the gradients' entry point, the other rows' outputs and sums being the same: the output's own rows are rounded
    against a largest weight that may be up to 2^8, and when it is taken anew depends on their neighbours."""
    n, heads, kv, dim = 300, 4, 2, 64
    q, k, v, dout = (normal((n, h, dim), dtype, i) for i, h in enumerate((heads, kv, kv, heads)))
    L, scale, at = binding.lib(), dim ** -0.5, 133
    rows = lambda *tensors: [op._heads(t, "t") for t in tensors]  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream

    def forward(q):
        out, lse = torch.empty_like(q), torch.empty(n, heads, device="cuda")
        binding.check(L.sllm_attention(*rows(q, k, v), None, window or 0, sinks, scale, *rows(out), lse.data_ptr(), 0, stream))
        return out, lse

    def gradients(q, out, lse):
        grads = [torch.empty_like(t) for t in (q, k, v)]
        size = op._workspace(L.sllm_attention_grad_workspace, *rows(q, k), None, window or 0, sinks)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        binding.check(L.sllm_attention_grad(*rows(dout, q, k, v, out), lse.data_ptr(), None, window or 0, sinks, scale, *rows(*grads),
                                            ws.data_ptr(), size, 0, stream))
        return grads

    out, lse = forward(q)
    clean = gradients(q, out, lse)
    far = q.clone()
    far[at] *= 3000
    far_out, far_lse = forward(far)
    assert (far_lse[at].abs() > 1000).any()
    out[at], lse[at] = far_out[at], far_lse[at]
    got = gradients(far, out, lse)
    rest = [i for i in range(n) if i != at]
    assert torch.equal(got[0][rest], clean[0][rest]) and all(torch.isfinite(t).all() for t in got)
    hidden = [j for j in range(n) if j > at or (window is not None and at - j >= window and j >= sinks)]
    for i in (1, 2):
        assert torch.equal(got[i][hidden], clean[i][hidden])
