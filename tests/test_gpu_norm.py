"""Norms, MX FP8 and products of it against the oracle's 64-bit definitions.

Tolerances, with u half a step of the type and e = 2^-24: a mean of squares of n columns in
32 bits is off by at most 2 (n + 8) e of itself, its root and inverse by half of that and 4 e
more; a norm multiplies twice, 2 e.  Gradients: a dot product over n columns is off by
2 (n + 8) e of the sum of its products' magnitudes.  A gain's gradient sums over rows.  In MX FP8
norms are held in 64 bits: codes and scales have to be equal, and so have quantised ones.

Products of MX FP8 in 16 bits: within each eight neighbouring columns products are added to
within 2^-13 of the largest, so they are off by 8 times that at the most; the sums of those are of 32
bits.  In 32 bits: as the products of a bfloat16 x.
"""

import math

import numpy as np
import pytest

from oracle import layer_oracle as O
from oracle import operators_oracle as O4
from tests.test_gpu_operators import SMALLEST, TYPES, UNIT, assert_close, host, normal, random_mx4, sum_bound

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import binding, operators as op  # noqa: E402

E = 2.0 ** -24


@pytest.fixture(autouse=True)
def _device(gpu_device):
    return gpu_device


SHAPES = [(1, 1), (1, 64), (3, 7), (5, 31), (2, 96), (70, 512), (9, 1000), (1025, 1096), (1500, 1500), (2, 2048), (3, 2049), (4, 4096),
          (2, 5120), (3, 8191), (2, 8200), (2, 16384), (3, 20001), (1, 32768), (2, 33000)]


def rounded(x, dtype):
    return host(torch.from_numpy(x).to(dtype))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_and_gradients(rows, cols, dtype, residual):
    gain_type = TYPES[(rows + cols) % 3]
    x = normal((rows, cols), dtype, cols, 2.0)
    r = normal((rows, cols), dtype, cols + 1) if residual else None
    gain = (1 + normal((cols,), torch.float32, 3, 0.2)).to(gain_type)
    dy, dh = normal((rows, cols), dtype, 4, 0.1), normal((rows, cols), dtype, 5, 0.1)
    leaves = [t.detach().requires_grad_() for t in (x, gain) + ((r,) if residual else ())]
    got = op.rms_norm(leaves[0], leaves[1], residual=leaves[2] if residual else None, eps=1e-4)
    y, h = got if residual else (got, x)
    # h is the rounded sum, exactly: 32 bits hold more than the sum of two 16-bit numbers needs, or round once
    want_h = (x.float() + r.float()).to(dtype) if residual else x
    assert torch.equal(h.detach(), want_h)
    hv, gv = host(want_h), host(gain)
    want = O.norm(hv, gv, 1e-4)
    rel = (cols + 16) * E
    assert_close(y, want, rel * np.abs(want), dtype)
    if residual:
        grads = torch.autograd.grad((y, h), leaves, (dy, dh))
        assert torch.equal(grads[0], grads[2])
    else:
        grads = torch.autograd.grad(y, leaves, dy)
    dyv, dhv = host(dy), host(dh) if residual else 0.0 * hv
    dx, dgain = O.norm_grad(dyv, dhv, hv, gv, 1e-4)
    f = 1 / np.sqrt((hv * hv).mean(1, keepdims=True) + 1e-4)
    size = np.abs(dhv) + f * (np.abs(dyv * gv) + np.abs(hv) * f * f * np.abs(dyv * gv * hv).mean(1, keepdims=True))
    assert_close(grads[0], dx, 5 * rel * size, dtype)
    assert_close(grads[1], dgain, (rel + 2 * (rows + 8) * E) * np.abs(dyv * hv * f).sum(0), gain_type)


@pytest.mark.parametrize("dtype", TYPES)
def test_one_of_two_gradients(dtype):
    """The norm or h alone used further; one leaf of three."""
    x, r = normal((6, 200), dtype, 1).requires_grad_(), normal((6, 200), dtype, 2).requires_grad_()
    gain = (1 + normal((200,), torch.float32, 3, 0.2)).requires_grad_()
    w = normal((6, 200), dtype, 4)
    y, h = op.rms_norm(x, gain, residual=r)
    both = torch.autograd.grad((y, h), (x, r, gain), (w, torch.zeros_like(w)), retain_graph=True)
    alone = torch.autograd.grad(y, (x, r, gain), w, retain_graph=True)
    for a, b in zip(both, alone):
        assert torch.equal(a, b)
    dx, dr, dg = torch.autograd.grad(h, (x, r, gain), w, allow_unused=True, retain_graph=True)
    assert torch.equal(dx, w) and torch.equal(dr, w) and (dg is None or not dg.any())
    (only,) = torch.autograd.grad(y, gain, w)
    assert torch.equal(only, alone[2])
    (s,) = torch.autograd.grad(op.rms_norm(x, gain.detach()).sum(), x)  # a gradient with strides of zero
    (t,) = torch.autograd.grad(op.rms_norm(x, gain.detach()), x, torch.ones_like(x))
    assert torch.equal(s, t)
    y, h = op.rms_norm(x, gain, residual=r)
    with torch.no_grad():
        gain += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Rows apart and starting anywhere, three dimensions, empty ones."""
    wide = normal((9, 333), dtype, 1)
    gain = 1 + normal((300,), torch.float32, 2, 0.1)
    want = op.rms_norm(wide[:, 5:305].contiguous(), gain)
    for got in (op.rms_norm(wide[:, 5:305], gain), op.rms_norm(wide[:, 5:305].contiguous().view(3, 3, 300), gain).view(9, 300)):
        assert (got.float() - want.float()).abs().max() <= 2 * UNIT[dtype] * want.float().abs().max()
    y, h = op.rms_norm(wide[:, 5:305], gain, residual=wide[:, 1:301])
    assert torch.equal(h, (wide[:, 5:305].float() + wide[:, 1:301].float()).to(dtype)) and y.is_contiguous() and h.is_contiguous()
    for shape in ((0, 8), (3, 0)):
        x = torch.empty(shape, dtype=dtype, device="cuda", requires_grad=True)
        g = torch.ones(shape[1], device="cuda", requires_grad=True)
        a, b = torch.autograd.grad(op.rms_norm(x, g).sum(), (x, g))
        assert a.shape == x.shape and b.shape == g.shape and not b.any()
    one = op.rms_norm(wide[0, 5:305], gain)
    assert one.shape == (300,)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_zero_or_not_finite(dtype):
    x = normal((5, 100), dtype, 1)
    x[1] = 0
    x[2, 7], x[3, 9] = math.nan, math.inf
    gain = torch.ones(100, device="cuda")
    y = op.rms_norm(x, gain)
    assert not y[1].any() and y[2].isnan().all() and torch.isfinite(y[[0, 4]]).all() and y[3, 9].isnan()
    q = op.rms_norm(x, gain, mx8=True)
    v = op.mx8_dequantize(q, torch.float32)
    assert not v[1].any() and v[2].isnan().all() and torch.isfinite(v[[0, 4]]).all()
    assert not op.rms_norm(torch.zeros(2, 100, dtype=dtype, device="cuda"), gain, eps=1e-6).any()


# ---- MX FP8 -----------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_in_eight_bits(rows, cols, dtype):
    rows = min(rows, 40)
    x, r = normal((rows, cols), dtype, cols, 2.0), normal((rows, cols), dtype, cols + 1)
    gain = (1 + normal((cols,), torch.float32, 3, 0.2))
    for residual in (None, r):
        got = op.rms_norm(x, gain, residual=residual, eps=1e-5, mx8=True)
        q, h = (got, x) if residual is None else got
        want_h = x if residual is None else (x.float() + r.float()).to(dtype)
        assert torch.equal(h, want_h)
        codes, scales = O.quantize8(O.norm(host(want_h), host(gain), float(np.float32(1e-5))))
        assert (q.codes.cpu().numpy() == codes).all() and (q.scales.cpu().numpy() == scales).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 33), (5, 127), (4, 512), (3, 513), (17, 768), (2, 1000), (33, 2051)])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize8(rows, cols, dtype):
    x = normal((rows, cols), dtype, rows + cols, 0.3) * torch.logspace(-6, 3, cols, device="cuda").to(dtype)
    q = op.mx8_quantize(x)
    codes, scales = O.quantize8(host(x))
    assert (q.codes.cpu().numpy() == codes).all() and (q.scales.cpu().numpy() == scales).all()
    want = O.dequantize8(codes, scales, cols)
    for to in TYPES:
        ref = torch.from_numpy(want).to(torch.float32).to(to)  # 64 to 32 bits is exact here
        assert torch.equal(op.mx8_dequantize(q, to).cpu(), ref)
    strided = torch.empty(rows, cols + 3, dtype=dtype, device="cuda")[:, 1:1 + cols]
    strided.copy_(x)
    again = op.mx8_quantize(strided, out=op.Mx8.empty(rows, cols, "cuda"))
    assert torch.equal(again.codes, q.codes) and torch.equal(again.scales, q.scales)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize8_edges(dtype):
    """Every bfloat16 pattern, in blocks of neighbours; for the other types what they make of them."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).to(dtype).view(-1, 64)
    q = op.mx8_quantize(x.cuda())
    codes, scales = O.quantize8(host(x))
    assert (q.scales.cpu().numpy() == scales).all() and (q.codes.cpu().numpy() == codes).all()


def test_dequantize8_every_code_and_scale():
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(8, 32), (256, 1))
    scales = np.zeros((2048, 16), np.uint8)
    scales[:, 0] = np.repeat(np.arange(256), 8)
    q = op.Mx8(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 32)
    want = torch.from_numpy(O.dequantize8(codes, scales, 32)).to(torch.float32)
    for to in TYPES:
        got, ref = op.mx8_dequantize(q, to).cpu(), want.to(to)
        assert ((got == ref) | (got.isnan() & ref.isnan())).all()


def random_mx8(rows, cols, seed, scales=(110, 128)):
    rng = np.random.default_rng(seed)
    blocks = -(-cols // 32)
    codes = rng.integers(0, 256, (rows, blocks * 32), dtype=np.uint8)
    codes[(codes & 127) == 127] = 0
    codes[:, cols:] = 0
    s = np.zeros((rows, -(-blocks // 16) * 16), np.uint8)
    s[:, :blocks] = rng.integers(*scales, (rows, blocks))
    return op.Mx8(torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), cols), O.dequantize8(codes, s, cols)


def grouped_bound(a, b):
    """8 times 2^-13 of the largest product of each eight columns, for a (m, k) times b (n, k)."""
    pad = -a.shape[1] % 8
    a, b = (np.pad(np.abs(t), ((0, 0), (0, pad))).reshape(len(t), -1, 8) for t in (a, b))
    bound = np.zeros((len(a), len(b)))
    for g in range(a.shape[1]):
        top = np.zeros_like(bound)
        for c in range(8):
            np.maximum(top, np.outer(a[:, g, c], b[:, g, c]), out=top)
        bound += 8 * 2.0 ** -13 * top
    return bound


PRODUCTS = [(1, 1, 1), (1, 200, 320), (3, 33, 64), (16, 200, 1000), (16, 30, 33), (17, 200, 320), (40, 513, 65), (128, 128, 512), (130, 257, 545),
            (300, 300, 96), (700, 129, 1100), (5, 1, 4100), (1, 2, 16000)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear8(m, n, k):
    x, xv = random_mx8(m, k, m + k)
    w, wv = random_mx4(n, k, n + k)
    want = O4.linear(xv, wv)
    sums = sum_bound(xv, wv.T, k)
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), want, sums, torch.float32)
    bound = sums + grouped_bound(xv, wv)
    y = op.mx4_linear(x, w)
    assert_close(y, want, bound, torch.bfloat16)
    if np.abs(want).max() < 60000:
        assert_close(op.mx4_linear(x, w, out_dtype=torch.float16), want, bound, torch.float16)
    out = torch.empty(m, n + 5, dtype=torch.bfloat16, device="cuda")[:, 2:2 + n]
    assert torch.equal(op.mx4_linear(x, w, out=out), y)


@pytest.mark.parametrize("m,n,k", [(300, 2100, 600), (2600, 4200, 96), (520, 8300, 1100)])
def test_linear8_of_large_tiles(m, n, k):
    x, xv = random_mx8(m, k, 1, (120, 128))
    w, wv = random_mx4(n, k, 2, (120, 128))
    rows, cols = np.r_[0:70, m - 70:m], np.r_[0:70, n - 70:n]
    got = op.mx4_linear(x, w)
    want = O4.linear(xv[rows], wv[cols])
    assert_close(got[torch.from_numpy(rows).cuda()][:, torch.from_numpy(cols).cuda()], want,
                 sum_bound(xv[rows], wv[cols].T, k) + grouped_bound(xv[rows], wv[cols]), torch.bfloat16)
    small = op.mx4_linear(x[m - 40:], w[n - 130:], out_dtype=torch.float32)
    assert_close(small, O4.linear(xv[m - 40:], wv[n - 130:]), sum_bound(xv[m - 40:], wv[n - 130:].T, k), torch.float32)


@pytest.mark.parametrize("m,n,k", [(3, 40, 200), (40, 300, 200), (300, 300, 700)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_linear8_with_nan_blocks(m, n, k, out):
    x, xv = random_mx8(m, k, 1, (120, 128))
    w, wv = random_mx4(n, k, 2, (120, 128))
    x.scales[m // 2, (k - 1) // 32] = 255
    w.scales[n // 2, 1] = 255
    y = op.mx4_linear(x, w, out_dtype=out).float().cpu().numpy()
    nan = np.zeros((m, n), bool)
    nan[m // 2] = nan[:, n // 2] = True
    assert (np.isnan(y) == nan).all()


def test_refusals():
    x, gain = normal((4, 64), torch.bfloat16, 1), torch.ones(64, device="cuda")
    for args in ((x, gain[:63]), (x, gain.view(1, 64)), (x.int(), gain), (x, gain.int()), (x.cpu(), gain), (x, gain.cpu()), (x[:, ::2], gain[:32]),
                 (x.t(), gain[:4])):
        with pytest.raises((ValueError, binding.SllmError)):
            op.rms_norm(*args)
    for more in ({"residual": x[:3]}, {"residual": x.float()}, {"residual": x.cpu()}, {"eps": -1.0}, {"eps": math.nan}):
        with pytest.raises((ValueError, binding.SllmError)):
            op.rms_norm(x, gain, **more)
    with pytest.raises(ValueError):
        op.rms_norm(x.clone().requires_grad_(), gain, mx8=True)
    with pytest.raises(ValueError):
        op.mx8_quantize(x.clone().requires_grad_())
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError):
            op.rms_norm(torch.autograd.forward_ad.make_dual(x, x), gain)
    q, w = op.mx8_quantize(x), op.mx4_quantize(x)
    for args in ((op.mx8_quantize(x[:, :32]), w), (q, op.mx4_quantize(x[:, :32]))):
        with pytest.raises((ValueError, binding.SllmError)):
            op.mx4_linear(*args)
    with pytest.raises((ValueError, AttributeError, binding.SllmError)):
        op.mx8_quantize(x, out=w)
    with pytest.raises(ValueError):
        op.mx8_dequantize(w)


def test_same_bytes_in_streams_and_graphs():
    """A norm in eight bits and its product, and a gradient, as one run of calls: eager, on
    streams of their own, and replayed from a graph while the inputs change."""
    x, r = normal((300, 1000), torch.bfloat16, 1), normal((300, 1000), torch.bfloat16, 2)
    gain = 1 + normal((1000,), torch.float32, 3, 0.1)
    w = op.mx4_quantize(normal((700, 1000), torch.bfloat16, 4, 0.02))
    dy = normal((300, 1000), torch.bfloat16, 5)

    def run(stream=None):
        y, h = op.rms_norm(x, gain, residual=r, mx8=True, stream=stream)
        z, _ = op.rms_norm(x, gain, residual=r, stream=stream)
        return op.mx4_linear(y, w, stream=stream), op.mx4_linear(y, w, out_dtype=torch.float32, stream=stream), h, z

    def gradient():
        leaves = [t.detach().requires_grad_() for t in (x, gain)]
        return torch.autograd.grad(op.rms_norm(*leaves), leaves, dy)

    want, first = run(), gradient()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        for _ in range(2):
            got = run(s)
            s.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)
    for a, b in zip(gradient(), first):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = run()
    for step in range(3):
        x.copy_(normal(x.shape, torch.bfloat16, 20 + step))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(run(), held):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,power", [(torch.float32, 100), (torch.float32, -100), (torch.bfloat16, 110), (torch.bfloat16, -90), (torch.float16, 13),
                                         (torch.float16, -12)])
@pytest.mark.parametrize("cols", [5, 1024, 4100, 17000, 33000])
def test_rows_whose_squares_leave_32_bits(cols, dtype, power):
    """Large or small all over, eps 0: a power of two times an ordinary row has its norm, and that power's inverse times its gradient."""
    u = normal((4, cols), dtype, cols).float().clamp(-4, 4)
    u = torch.where(u.abs() < 2.0 ** -2, 0.25, u)  # nothing of it becomes subnormal
    x = (u * 2.0 ** power).to(dtype).requires_grad_()
    gain = (1 + normal((cols,), torch.float32, 3, 0.2)).requires_grad_()
    dy = normal((4, cols), dtype, 4, 0.1)
    y = op.rms_norm(x, gain, eps=0.0)
    y.backward(dy)
    xv, gv, dyv = host(x), host(gain), host(dy)
    want = O.norm(xv, gv, 0.0)
    rel = (cols + 16) * E
    assert_close(y, want, rel * np.abs(want), dtype)
    dx, dgain = O.norm_grad(dyv, 0 * xv, xv, gv, 0.0)
    f = 1 / np.sqrt((xv * xv).mean(1, keepdims=True))
    size = f * (np.abs(dyv * gv) + np.abs(xv) * f * f * np.abs(dyv * gv * xv).mean(1, keepdims=True))
    if dtype == torch.float16 and power < 0:  # gradients of its inverse: some past the type's largest
        dx = np.where(np.abs(dx) < 65000, dx, 0)
        x.grad[torch.from_numpy(dx == 0).to(x.grad.device)] = 0
    assert_close(x.grad, dx, 5 * rel * size, dtype)
    assert_close(gain.grad, dgain, (rel + 24 * E) * np.abs(dyv * xv * f).sum(0), torch.float32)


@pytest.mark.parametrize("rows,cols", [(15, 8), (17, 128), (33, 129), (40000, 64), (32769, 33), (5, 512), (9001, 257), (2, 513)])
@pytest.mark.parametrize("dtype", TYPES)
def test_short_rows(rows, cols, dtype):
    """Heads as rows: many side by side, the last workgroup's not all there."""
    for residual in (False, True):
        test_norm_and_gradients(rows, cols, dtype, residual)
    q = op.rms_norm(normal((rows, cols), dtype, 1), torch.ones(cols, device="cuda"), mx8=True)
    codes, scales = O.quantize8(O.norm(host(normal((rows, cols), dtype, 1)), np.ones(cols), float(np.float32(1e-5))))
    assert (q.codes.cpu().numpy() == codes).all() and (q.scales.cpu().numpy() == scales).all()


@pytest.mark.parametrize("m,n,k", [(18, 1, 1), (32, 17, 33), (31, 513, 1100), (25, 100, 4100), (32, 1025, 545), (33, 64, 64)])
def test_products_of_two_sixteens_of_rows(m, n, k):
    test_linear8(m, n, k)
