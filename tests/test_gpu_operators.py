"""The operators on loaded weights against the oracle's 64-bit definitions.

Tolerances.  A sum of `depth` products in 32 bits, whatever its order, is off
by at most about depth * 2^-24 times the sum of the products' magnitudes; twice
that, and eight terms more for the joins, is allowed (`sum_bound`).  Rounding
to the output's type then adds half a unit in its last place: 2^-8 of the
value for bfloat16, 2^-11 for float16, 2^-24 for float32, and half of the
smallest step for float16's subnormals (2^-25).  Quantised codes and scales,
dequantised values and lookups with a scale that is a power of two have to be
equal.
"""

import math

import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import binding, operators as op  # noqa: E402

TYPES = [torch.bfloat16, torch.float16, torch.float32]
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}


@pytest.fixture(autouse=True)
def _device(gpu_device):
    return gpu_device


def host(t):
    return t.detach().double().cpu().numpy()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def sum_bound(a, b, depth):
    """What a sum in 32 bits may be off by, for a (m, depth) times b (depth, n)."""
    return 2 * (depth + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(b))


def assert_close(got, want, bound, dtype):
    assert got.dtype == dtype
    g = host(got)
    assert g.shape == want.shape
    tol = bound + (np.abs(want) + bound) * UNIT[dtype] + SMALLEST[dtype]
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: " \
                          f"{g[bad][0]} for {want[bad][0]}, allowed {np.broadcast_to(tol, bad.shape)[bad][0]}"


def random_mx4(rows, cols, seed, scales=(110, 128)):
    """Every code and scales of a range; padded columns and bytes as the format has them."""
    rng = np.random.default_rng(seed)
    blocks = -(-cols // 32)
    codes = rng.integers(0, 256, (rows, blocks * 16), dtype=np.uint8)
    if cols % 32:
        code = np.stack([codes & 15, codes >> 4], -1).reshape(rows, -1)
        code[:, cols:] = 0
        codes = code[:, 0::2] | (code[:, 1::2] << 4)
    s = np.zeros((rows, -(-blocks // 16) * 16), np.uint8)
    s[:, :blocks] = rng.integers(*scales, (rows, blocks))
    return op.Mx4(torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), cols), O.dequantize(codes, s, cols)


# ---- quantisation -----------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 127), (4, 128), (7, 512), (3, 513), (17, 768),
                                       (2, 1000), (64, 96), (1, 4096), (33, 2051)])
def test_quantize(dtype, rows, cols):
    x = normal((rows, cols), dtype, rows * 1000 + cols, 0.02)
    q = op.mx4_quantize(x)
    codes, scales = O.quantize(host(x))
    assert (q.scales.cpu().numpy() == scales).all()
    assert (q.codes.cpu().numpy() == codes).all()
    back = op.mx4_dequantize(q, torch.float32)
    assert (host(back) == O.dequantize(codes, scales, cols)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_edges(dtype):
    """Ties, zeros, the largest and smallest magnitudes, infinities and NaN."""
    x = torch.zeros(16, 96, dtype=torch.float32)
    x[0, :16] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -7.5])
    x[1, 5] = math.inf
    x[2, 40] = -math.inf
    x[3, 95] = math.nan
    x[4] = torch.finfo(dtype).max
    x[5] = torch.finfo(dtype).tiny
    x[6, :4] = torch.tensor([1.0, 2.0 ** -20, -2.0 ** -24, 3e-7])
    x[7] = -0.0
    x[8] = torch.finfo(dtype).smallest_normal / 4
    x[9, 0], x[9, 1] = 3e-39, 1e-40
    x[10] = -torch.finfo(dtype).max
    x[11, 31], x[11, 32], x[11, 63] = 4.0, 3.9999, -8.0
    x = x.to(dtype)
    q = op.mx4_quantize(x.cuda())
    codes, scales = O.quantize(host(x))
    assert (q.scales.cpu().numpy() == scales).all()
    assert (q.codes.cpu().numpy() == codes).all()
    back, want = host(op.mx4_dequantize(q, torch.float32)), O.dequantize(codes, scales, 96)
    assert ((back == want) | (np.isnan(back) & np.isnan(want))).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_every_bfloat16_is_quantized_as_defined(dtype):
    """Each of the 2^16 bfloat16 patterns, in blocks of 32 neighbours and alone in its block."""
    if dtype != torch.bfloat16:
        bits = np.random.default_rng(3).integers(0, 1 << 32, 1 << 14, dtype=np.uint32)
        x = torch.from_numpy(bits.view(np.float32).copy()).to(dtype).view(-1, 64)
    else:
        x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(-1, 64)
    q = op.mx4_quantize(x.cuda())
    codes, scales = O.quantize(host(x))
    assert (q.scales.cpu().numpy() == scales).all() and (q.codes.cpu().numpy() == codes).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_dequantize_every_code_and_scale(dtype):
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(16, 16), (16, 1))
    codes = np.repeat(codes, 1, 0)
    scales = np.zeros((256, 16), np.uint8)
    scales[:, 0] = np.arange(256)
    want = O.dequantize(codes, scales, 32)
    q = op.Mx4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 32)
    got = op.mx4_dequantize(q, dtype).cpu()
    ref = torch.from_numpy(want).to(torch.float32).to(dtype)  # 64 to 32 bits is exact or infinite here
    assert ((got == ref) | (got.isnan() & ref.isnan())).all()


def test_quantize_strides_and_outputs():
    base = normal((40, 300), torch.bfloat16, 5)
    for x in (base[:, :256], base[::3, 5:201], base[1:2], base.view(8, 5, 300), base[7]):
        q = op.mx4_quantize(x)
        codes, scales = O.quantize(host(x.reshape(-1, x.shape[-1])))
        assert (q.codes.cpu().numpy() == codes).all() and (q.scales.cpu().numpy() == scales).all()
    q = op.Mx4.empty(10, 300, "cuda")
    q.codes.fill_(255)
    q.scales.fill_(255)
    assert op.mx4_quantize(base[:10], out=q) is q
    assert (q.scales.cpu().numpy() == O.quantize(host(base[:10]))[1]).all()  # padding bytes too
    out = torch.full((40, 320), 7.0, device="cuda")
    op.mx4_dequantize(op.mx4_quantize(base), out=out[:, 3:303])
    want = O.dequantize(*O.quantize(host(base)), 300)
    assert (host(out[:, 3:303]) == want).all() and (out[:, :3] == 7).all() and (out[:, 303:] == 7).all()


# ---- products ---------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 16, 32), (1, 768, 768), (2, 33, 65), (5, 1000, 129), (16, 64, 4096), (17, 130, 31), (33, 96, 544),
          (64, 256, 512), (65, 257, 1000), (100, 768, 1536), (128, 128, 128), (130, 70, 2051), (256, 512, 96),
          (300, 513, 640), (1, 2047, 5120), (513, 300, 333)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear(dtype, m, n, k):
    x = normal((m, k), dtype, m + n + k)
    w, wv = random_mx4(n, k, m * n + k)
    a = host(x)
    assert_close(op.mx4_linear(x, w), O.linear(a, wv), sum_bound(a, wv.T, k), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_mx(dtype, m, n, k):
    x, xv = random_mx4(m, k, m + n + k, (118, 130))
    w, wv = random_mx4(n, k, m * n + k)
    assert_close(op.mx4_linear(x, w, out_dtype=dtype), O.linear(xv, wv), sum_bound(xv, wv.T, k), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_grad(dtype, m, n, k):
    dy = normal((m, n), dtype, m + n + k, 0.1)
    w, wv = random_mx4(n, k, m * n + k)
    a = host(dy)
    assert_close(op.mx4_linear_grad(dy, w), O.linear_grad(a, wv), sum_bound(a, wv, n), dtype)


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32),
                                             (torch.float16, torch.float32)])
@pytest.mark.parametrize("m", [3, 200])
def test_linear_other_types(dtype, out_dtype, m):
    x, dy = normal((m, 288), dtype, 1), normal((m, 160), dtype, 2)
    w, wv = random_mx4(160, 288, 3)
    a, b = host(x), host(dy)
    assert_close(op.mx4_linear(x, w, out_dtype=out_dtype), O.linear(a, wv), sum_bound(a, wv.T, 288), out_dtype)
    assert_close(op.mx4_linear_grad(dy, w, out_dtype=out_dtype), O.linear_grad(b, wv), sum_bound(b, wv, 160), out_dtype)


@pytest.mark.parametrize("m", [1, 7, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_strides(dtype, m):
    """Rows apart by odd strides, starting off any wider alignment, into part of a larger output."""
    k, n = 200, 170
    base = normal((m, k + 37), dtype, 9)
    w, wv = random_mx4(n, k, 10)
    for first in (0, 1, 8):
        x = base[:, first:first + k]
        out = torch.full((m, n + 11), 3.0, dtype=dtype, device="cuda")
        op.mx4_linear(x, w, out=out[:, 5:5 + n])
        assert_close(out[:, 5:5 + n], O.linear(host(x), wv), sum_bound(host(x), wv.T, k), dtype)
        assert (out[:, :5] == 3).all() and (out[:, 5 + n:] == 3).all()
        dy = base[:, first:first + n]
        dx = torch.full((m, k + 9), 3.0, dtype=dtype, device="cuda")
        op.mx4_linear_grad(dy, w, out=dx[:, 1:1 + k])
        assert_close(dx[:, 1:1 + k], O.linear_grad(host(dy), wv), sum_bound(host(dy), wv, n), dtype)
        assert (dx[:, :1] == 3).all() and (dx[:, 1 + k:] == 3).all()


@pytest.mark.parametrize("m", [1, 40, 300])
def test_linear_empty(m):
    w, _ = random_mx4(64, 96, 1)
    assert op.mx4_linear(normal((0, 96), torch.bfloat16, 1), w).shape == (0, 64)
    assert op.mx4_linear_grad(normal((0, 64), torch.bfloat16, 1), w).shape == (0, 96)
    none = op.Mx4.empty(0, 96, "cuda")
    assert op.mx4_linear(normal((m, 96), torch.bfloat16, 1), none).shape == (m, 0)
    dx = op.mx4_linear_grad(torch.empty(m, 0, dtype=torch.bfloat16, device="cuda"), none)
    assert dx.shape == (m, 96) and not dx.any()
    thin = op.Mx4.empty(64, 0, "cuda")
    y = op.mx4_linear(torch.empty(m, 0, dtype=torch.bfloat16, device="cuda"), thin)
    assert y.shape == (m, 64) and not y.any()
    y = op.mx4_linear(op.Mx4.empty(m, 0, "cuda"), thin)
    assert y.shape == (m, 64) and not y.any()


@pytest.mark.parametrize("m", [1, 6, 40, 300])
def test_linear_not_finite(m):
    """A NaN or an infinity of x reaches its own row of the result, a NaN block of w its own column."""
    k, n = 320, 200
    x = normal((m, k), torch.bfloat16, 4)
    w, wv = random_mx4(n, k, 5)
    x[m - 1, k - 1] = math.inf
    y = op.mx4_linear(x, w)
    assert not y[m - 1].isfinite().any() or (wv[:, k - 1] == 0).any()
    assert y[:m - 1].isfinite().all()
    x[m - 1, k - 1] = math.nan
    y = op.mx4_linear(x, w)
    assert y[m - 1].isnan().all() and y[:m - 1].isfinite().all()
    x[m - 1, k - 1] = 1.0
    w.scales[n - 1, 9] = 255
    for y in (op.mx4_linear(x, w), op.mx4_linear(op.mx4_quantize(x), w)):
        assert y[:, n - 1].isnan().all() and y[:, :n - 1].isfinite().all()
    dx = op.mx4_linear_grad(normal((m, n), torch.bfloat16, 6), w)
    assert dx[:, 288:].isnan().all() and dx[:, :288].isfinite().all()
    # garbage in what the format leaves unused must not matter
    q = op.mx4_quantize(x)
    want = op.mx4_linear(q, w[:n - 1])
    q.scales[:, 10:] = 255
    w.scales[:, 10:] = 255
    assert torch.equal(op.mx4_linear(q, w[:n - 1]), want)
    assert torch.equal(op.mx4_linear(x, w[:n - 1]), y_first(x, w, n))


def y_first(x, w, n):
    clean = op.Mx4(w.codes[:n - 1].clone(), w.scales[:n - 1].clone(), w.cols)
    clean.scales[:, 10:] = 0
    return op.mx4_linear(x, clean)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_linear_keeps_the_precision_of_x(dtype):
    """Elements of more bits than bfloat16 holds are not cut."""
    k, n = 64, 48
    w, wv = random_mx4(n, k, 6, (127, 128))
    for m in (1, 20, 256):
        x = torch.zeros(m, k, dtype=dtype, device="cuda")
        x[:, 0] = 1 + (2.0 ** -10 if dtype == torch.float16 else 2.0 ** -23)
        a = host(x)
        got = host(op.mx4_linear(x, w, out_dtype=torch.float32))
        assert (got == (a @ wv.T).astype(np.float32)).all()
        dy = torch.zeros(m, n, dtype=dtype, device="cuda")
        dy[:, 3] = x[0, 0]
        got = host(op.mx4_linear_grad(dy, w, out_dtype=torch.float32))
        assert (got == (host(dy) @ wv).astype(np.float32)).all()


@pytest.mark.parametrize("m", [1, 9, 70, 260])
def test_linear_extreme_scales(m):
    """Blocks far apart in size: the small ones are lost only where 32 bits lose them."""
    w, wv = random_mx4(96, 128, 7, (20, 230))
    x = normal((m, 128), torch.bfloat16, 8)
    a = host(x)
    got = op.mx4_linear(x, w, out_dtype=torch.float32)
    assert_close(got, O.linear(a, wv), sum_bound(a, wv.T, 128), torch.float32)
    small, smallv = random_mx4(96, 128, 7, (0, 60))
    got = op.mx4_linear(x, small, out_dtype=torch.float32)
    assert_close(got, O.linear(a, smallv), sum_bound(a, smallv.T, 128) + 128 * 2.0 ** -149, torch.float32)


@pytest.mark.parametrize("m,n,k", [(70, 200, 320), (129, 130, 1100), (3300, 3600, 96), (3300, 96, 3600)])
@pytest.mark.parametrize("scale", [0, 30, 95, 96, 132, 133, 180])
def test_linear_half_any_scale(m, n, k, scale):
    """x in float16 against blocks whose values float16 holds, scaled or not, and one that it may not."""
    w, wv = random_mx4(n, k, 15, (96, 133))
    x, dy = normal((m, k), torch.float16, 16), normal((m, n), torch.float16, 17)
    x[0, :] = 2.0 ** -24  # the smallest
    x[m - 1, ::2] = 2.0 ** -15
    dy[0, :] = -2.0 ** -24
    for row, block in ((n - 1, (k - 1) // 32), (n // 2, 1)):
        w.scales[row, block] = scale
        wv = O.dequantize(w.codes.cpu().numpy(), w.scales.cpu().numpy(), k)
        a, b = host(x), host(dy)
        assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, k), torch.float32)
        assert_close(op.mx4_linear_grad(dy, w, out_dtype=torch.float32), O.linear_grad(b, wv), sum_bound(b, wv, n), torch.float32)
    w.scales[n - 1, 0] = 255
    y = op.mx4_linear(x, w, out_dtype=torch.float32)
    assert y[:, n - 1].isnan().all() and y[:, :n - 1].isfinite().all()
    dx = op.mx4_linear_grad(dy, w, out_dtype=torch.float32)
    assert dx[:, :32].isnan().all() and dx[:, 32:].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(4, 33000), (5, 33000), (16, 8200), (16, 17000), (17, 8200), (32, 8200), (33, 8200), (64, 300),
                                 (65, 300), (128, 300), (129, 300)])
def test_linear_around_row_limits(dtype, m, n):
    """Where the way of carrying out a product changes with its rows and columns."""
    k = 160
    w, wv = random_mx4(n, k, m)
    x = normal((m, k), dtype, 21)
    a = host(x)
    assert_close(op.mx4_linear(x, w), O.linear(a, wv), sum_bound(a, wv.T, k), dtype)
    q = op.mx4_quantize(x)
    a = host(op.mx4_dequantize(q, torch.float32))
    assert_close(op.mx4_linear(q, w, out_dtype=dtype), O.linear(a, wv), sum_bound(a, wv.T, k), dtype)


@pytest.fixture(scope="module", params=[(130, 2100, 8200), (50, 4300, 8200), (3300, 3600, 96), (3300, 96, 3600)],
                ids=lambda s: "x".join(map(str, s)))
def large_weight(request):
    m, n, k = request.param
    return (m, n, k) + random_mx4(n, k, 23)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_every_tile(large_weight, dtype):
    """Problems that go by the tallest tiles of each kind, with rows and columns past the last whole one."""
    m, n, k, w, wv = large_weight
    x, dy = normal((m, k), dtype, 24), normal((m, n), dtype, 25)
    a, b = host(x), host(dy)
    assert_close(op.mx4_linear(x, w), O.linear(a, wv), sum_bound(a, wv.T, k), dtype)
    assert_close(op.mx4_linear_grad(dy, w), O.linear_grad(b, wv), sum_bound(b, wv, n), dtype)
    q = op.mx4_quantize(x)
    a = host(op.mx4_dequantize(q, torch.float32))
    assert_close(op.mx4_linear(q, w, out_dtype=dtype), O.linear(a, wv), sum_bound(a, wv.T, k), dtype)


def test_linear_in_halves():
    """Large tiles with the depth in two, where float's three parts make it deep enough."""
    m, n, k = 1500, 4900, 2800
    w, wv = random_mx4(n, k, 26)
    x = normal((m, k), torch.float32, 27)
    assert_close(op.mx4_linear(x, w), O.linear(host(x), wv), sum_bound(host(x), wv.T, k), torch.float32)
    v, vv = random_mx4(k, n, 28)
    assert_close(op.mx4_linear_grad(x, v), O.linear_grad(host(x), vv), sum_bound(host(x), vv, k), torch.float32)


def test_linear_mx_in_halves():
    """The same with both sides in MX FP4, against the small tiles that 100 rows at a time go by: each is off by
    at most a sum's bound."""
    m, n, k = 1500, 4900, 8200
    w, _ = random_mx4(n, k, 29, (120, 124))
    q = op.mx4_quantize(normal((m, k), torch.float32, 30))
    whole = op.mx4_linear(q, w, out_dtype=torch.float32)
    parts = torch.cat([op.mx4_linear(q[r:r + 100], w, out_dtype=torch.float32) for r in range(0, m, 100)])
    sizes = op.mx4_dequantize(q, torch.float32).abs() @ op.mx4_dequantize(w, torch.float32).abs().T
    assert ((whole - parts).abs() <= 2 * 2 * (k + 8) * 2.0 ** -24 * sizes).all()


def test_linear_half_small_values():
    """A weight far below float16's range against large x: no value is lost."""
    m, n, k = 150, 140, 256
    w, wv = random_mx4(n, k, 18, (1, 60))
    x = normal((m, k), torch.float16, 19, 1000.0)
    dy = normal((m, n), torch.float16, 20, 1000.0)
    a, b = host(x), host(dy)
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, k), torch.float32)
    assert_close(op.mx4_linear_grad(dy, w, out_dtype=torch.float32), O.linear_grad(b, wv), sum_bound(b, wv, n), torch.float32)


def test_linear_same_bytes_again():
    for m in (1, 30, 200):
        x = normal((m, 4096), torch.bfloat16, 1)
        w, _ = random_mx4(512, 4096, 2)
        y, dx = op.mx4_linear(x, w), op.mx4_linear_grad(normal((m, 512), torch.bfloat16, 3), w)
        for _ in range(3):
            assert torch.equal(op.mx4_linear(x, w), y)
            assert torch.equal(op.mx4_linear_grad(normal((m, 512), torch.bfloat16, 3), w), dx)


def test_linear_rows_of_a_weight():
    """A run of rows is a weight of its own, and leading dimensions pass through."""
    w, wv = random_mx4(100, 96, 1)
    x = normal((2, 3, 96), torch.bfloat16, 2)
    a = host(x).reshape(6, 96)
    y = op.mx4_linear(x, w[13:77])
    assert y.shape == (2, 3, 64)
    assert_close(y.view(6, 64), O.linear(a, wv[13:77]), sum_bound(a, wv[13:77].T, 96), torch.bfloat16)
    y = op.mx4_linear(x[0, 0], w)
    assert y.shape == (100,)


# ---- embeddings -------------------------------------------------------------

def some_ids(n, vocab, dtype, seed, padding=True):
    g = gen(seed)
    ids = torch.exp(torch.rand(n, generator=g, device="cuda") * math.log(vocab)).long().clamp(max=vocab) - 1
    if padding and n > 2:
        ids[::7] = -1
        ids[3::11] = vocab
        if dtype == torch.int64:
            ids[5::13] = (1 << 32) + 1  # names no row, whatever its low half is
    return ids.to(dtype)


@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (3, 10, 7), (16, 1000, 768), (5, 50, 1001), (700, 33, 96), (2, 9, 8192),
                                         (1000, 500, 40)])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding(dtype, n, vocab, dim, ids_dtype):
    table = normal((vocab, dim), dtype, n)
    ids = some_ids(n, vocab, ids_dtype, dim)
    for scale in (1.0, 0.25, 3.3):
        f = float(np.float32(scale))
        want = O.embedding(host(table), ids.tolist(), f)
        assert_close(op.embedding(table, ids, scale), want, np.abs(want) * 2.0 ** -24, dtype)
        got = op.embedding(table, ids, scale, out_dtype=torch.float32)
        assert_close(got, want, 0 if scale != 3.3 else np.abs(want) * 2.0 ** -24, torch.float32)
        if scale != 3.3:
            assert (host(got) == want).all()


@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (3, 10, 7), (16, 100, 768), (300, 33, 97), (2, 9, 8192)])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_mx(dtype, n, vocab, dim):
    table, tv = random_mx4(vocab, dim, n)
    ids = some_ids(n, vocab, torch.int64, dim)
    for scale in (1.0, 2.7):
        want = O.embedding(tv, ids.tolist(), float(np.float32(scale)))
        assert_close(op.embedding(table, ids, scale, out_dtype=dtype), want, np.abs(want) * 2.0 ** -24, dtype)


def test_embedding_strides():
    base = normal((50, 333), torch.float16, 1)
    ids = some_ids(24, 50, torch.int32, 2).view(4, 6)
    table = base[:, 7:207]
    out = torch.full((24, 210), 5.0, dtype=torch.float16, device="cuda")
    op.embedding(table, ids.view(-1), 1.0, out=out[:, 3:203])
    want = O.embedding(host(table), ids.flatten().tolist(), 1.0)
    assert (host(out[:, 3:203]) == want).all() and (out[:, :3] == 5).all() and (out[:, 203:] == 5).all()
    assert op.embedding(table, ids).shape == (4, 6, 200)
    assert op.embedding(table, ids[:0]).shape == (0, 6, 200)


@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab,dim", [(0, 5, 8), (1, 1, 1), (3, 10, 7), (64, 1000, 768), (500, 50, 101), (1500, 3, 64),
                                         (2100, 4000, 130), (5000, 700, 32), (900, 1, 264), (4097, 100000, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_grad(dtype, n, vocab, dim, ids_dtype):
    dy = normal((n, dim), dtype, n + 1, 0.5)
    ids = some_ids(n, vocab, ids_dtype, dim)
    scale = float(np.float32(0.37))
    want = O.embedding_grad(host(dy), ids.tolist(), vocab, scale)
    size = O.embedding_grad(np.abs(host(dy)), ids.tolist(), vocab, scale)
    count = np.bincount([v for v in ids.tolist() if 0 <= v < vocab], minlength=vocab)[:, None]
    bound = 2 * (count + 8) * 2.0 ** -24 * size
    for out_dtype in {dtype, torch.float32}:
        assert_close(op.embedding_grad(dy, ids, vocab, 0.37, out_dtype=out_dtype), want, bound, out_dtype)


@pytest.mark.parametrize("n,vocab,dim", [(1, 4, 3), (700, 40, 96), (2000, 9, 257), (3000, 5000, 64)])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_grad_accumulates(dtype, n, vocab, dim):
    dy = normal((n, dim), torch.bfloat16, n)
    ids = some_ids(n, vocab, torch.int32, dim)
    base = torch.full((vocab, dim + 13), 2.0, dtype=dtype, device="cuda")
    grad = base[:, 5:5 + dim]
    grad.copy_(normal((vocab, dim), dtype, 3))
    before = grad.clone()
    want = O.embedding_grad(host(dy), ids.tolist(), vocab, 1.0, host(before))
    size = O.embedding_grad(np.abs(host(dy)), ids.tolist(), vocab, 1.0, np.abs(host(before)))
    got = op.embedding_grad(dy, ids, vocab, out=grad, accumulate=True)
    assert got is grad
    assert_close(grad, want, 2 * (n + 8) * 2.0 ** -24 * size, dtype)
    named = set(ids.tolist())
    rest = [v for v in range(vocab) if v not in named]
    assert torch.equal(grad[rest], before[rest])
    assert (base[:, :5] == 2).all() and (base[:, 5 + dim:] == 2).all()


def test_embedding_grad_same_bytes_again():
    """Sums run in the order of positions: nothing depends on which wave came first."""
    dy = normal((6000, 200), torch.float32, 1)
    ids = some_ids(6000, 300, torch.int64, 2)
    first = op.embedding_grad(dy, ids, 300)
    for _ in range(5):
        assert torch.equal(op.embedding_grad(dy, ids, 300), first)


def test_embedding_grad_strides():
    base = normal((40, 333), torch.bfloat16, 1)
    ids = some_ids(40, 30, torch.int64, 2).view(5, 8)
    dy = base[:, 3:203].unflatten(0, (5, 8))
    want = O.embedding_grad(host(dy).reshape(40, 200), ids.flatten().tolist(), 30, 1.0)
    size = O.embedding_grad(np.abs(host(dy)).reshape(40, 200), ids.flatten().tolist(), 30, 1.0)
    out = torch.full((30, 202), 9.0, device="cuda")
    op.embedding_grad(dy, ids, 30, out=out[:, 1:201])
    assert_close(out[:, 1:201], want, 96 * 2.0 ** -24 * size, torch.float32)
    assert (out[:, 0] == 9).all() and (out[:, 201] == 9).all()


# ---- gradients, streams, graphs, refusals -----------------------------------

def test_autograd():
    w, wv = random_mx4(48, 64, 1)
    table = normal((20, 64), torch.float32, 2).requires_grad_()
    ids = some_ids(9, 20, torch.int64, 3)
    y = op.mx4_linear(op.embedding(table, ids, 0.5), w)
    y.sum().backward()  # its gradient has strides of 0
    want = O.embedding_grad(O.linear_grad(np.ones((9, 48)), wv), ids.tolist(), 20, 0.5)
    size = O.embedding_grad(O.linear_grad(np.ones((9, 48)), np.abs(wv)), ids.tolist(), 20, 0.5)
    assert_close(table.grad, want, 4 * (48 + 9 + 8) * 2.0 ** -24 * size, torch.float32)
    # against differences of the forward pass: it is linear, so a step of any size serves
    step = normal((20, 64), torch.float32, 4)
    with torch.no_grad():
        plus = op.mx4_linear(op.embedding(table + step, ids, 0.5), w).double().sum()
        minus = op.mx4_linear(op.embedding(table - step, ids, 0.5), w).double().sum()
    diff = float(plus - minus) / 2
    scale = float((step.abs().double() * torch.from_numpy(size).cuda()).sum())
    weight = float(np.abs(host(table)).max() + 1) * size.sum()
    assert abs(diff - float((step.double() * table.grad.double()).sum())) <= (scale + weight) * 200 * 2.0 ** -24
    with pytest.raises(ValueError):
        op.mx4_linear(table, w, out=torch.empty(20, 48, device="cuda"))


def test_streams():
    s = torch.cuda.Stream()
    x = normal((300, 512), torch.bfloat16, 1)
    w, _ = random_mx4(256, 512, 2)
    ids = some_ids(300, 100, torch.int64, 3)
    want = (op.mx4_linear(x, w), op.mx4_linear_grad(op.mx4_linear(x, w), w), op.embedding_grad(x, ids, 100),
            op.mx4_linear(op.mx4_quantize(x), w))
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        y = op.mx4_linear(x, w, stream=stream)
        got = (y, op.mx4_linear_grad(y, w, stream=stream), op.embedding_grad(x, ids, 100, stream=stream),
               op.mx4_linear(op.mx4_quantize(x, stream=stream), w, stream=stream))
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("m", [1, 64, 300])
def test_graph_replays(m):
    """Captured calls, replayed over new inputs with other work in between, give the eager results."""
    x = normal((m, 1024), torch.float16, 1)
    w, _ = random_mx4(512, 1024, 2)
    ids = some_ids(m, 90, torch.int64, 3, padding=False)

    def step():
        q = op.mx4_quantize(x)
        y = op.mx4_linear(x, w)
        return y, op.mx4_linear(q, w), op.mx4_linear_grad(y, w), op.embedding(w, ids, 2.0), op.embedding_grad(x, ids, 90)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        x.copy_(normal((m, 1024), torch.float16, 10 + seed))
        ids.copy_(some_ids(m, 90, torch.int64, 20 + seed, padding=seed % 2 == 1))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b)


def test_calls_in_python(monkeypatch):
    """The calls that the extension does not make, and all of them without it, have the same results and refusals."""
    w, _ = random_mx4(130, 96, 41)
    ids = some_ids(300, 50, torch.int64, 42)
    table = normal((50, 96), torch.float16, 43)
    x, dy = normal((2, 3, 96), torch.bfloat16, 44), normal((2, 3, 130), torch.float32, 45)
    wide = normal((6, 200), torch.bfloat16, 46)

    def results():
        q = op.mx4_quantize(x)
        yield q.codes
        yield q.scales
        yield op.mx4_dequantize(q, torch.float16)
        yield op.mx4_linear(x, w)
        yield op.mx4_linear(x, w, out_dtype=torch.float32)
        yield op.mx4_linear(x[0, 0], w)
        yield op.mx4_linear(wide[:, 7:103], w)
        yield op.mx4_linear(q, w)
        yield op.mx4_linear_grad(dy, w, out_dtype=torch.float16)
        yield op.embedding(table, ids, scale=0.5)
        yield op.embedding(table, ids.view(20, 15).int())
        yield op.embedding(w, ids, out_dtype=torch.float32)
        yield op.embedding_grad(normal((300, 96), torch.float32, 47), ids, 50, scale=2.0, out_dtype=torch.bfloat16)
        yield op.mx4_linear(x[:, :0], w)

    def refusals():
        for call in (lambda: op.mx4_linear(x[..., :64], w), lambda: op.mx4_linear(x.transpose(0, 2), w),
                     lambda: op.mx4_linear(x, w, out_dtype=torch.float64), lambda: op.mx4_linear(x.double(), w),
                     lambda: op.mx4_linear(x.cpu(), w), lambda: op.mx4_quantize(x.double()),
                     lambda: op.mx4_dequantize(w, torch.int8), lambda: op.embedding(table, ids.float()),
                     lambda: op.embedding(table, ids.cpu()), lambda: op.embedding(x, ids),
                     lambda: op.embedding_grad(dy, ids, 50), lambda: op.mx4_linear_grad(x, w)):
            with pytest.raises((ValueError, binding.SllmError)) as e:
                call()
            yield str(e.value)

    assert op._native() is not None
    native, said = list(results()), list(refusals())
    monkeypatch.setattr(op, "_native", lambda: None)
    for a, b in zip(native, list(results()), strict=True):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)
    assert said == list(refusals())


def test_refusals():
    w, _ = random_mx4(64, 96, 1)
    x = normal((4, 96), torch.bfloat16, 2)
    out = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        op.mx4_linear(x.double(), w)
    with pytest.raises(ValueError):
        op.mx4_linear(x.t(), w)
    with pytest.raises(ValueError):
        op.mx4_linear(x, w, out=out[:, :63])
    with pytest.raises(ValueError):
        op.mx4_linear(x.cpu(), w)
    with pytest.raises(binding.SllmError):
        op.mx4_linear(x[:, :64], w)
    with pytest.raises(binding.SllmError):
        op.mx4_linear_grad(x, w)
    with pytest.raises(binding.SllmError):  # rows that overlap
        op.mx4_linear(torch.zeros(200, dtype=torch.bfloat16, device="cuda").as_strided((4, 96), (8, 1)), w)
    square, _ = random_mx4(96, 96, 1)
    with pytest.raises(binding.SllmError) as e:  # the output overlaps the input
        op.mx4_linear(x, square, out=x)
    assert e.value.code == -1
    with pytest.raises(binding.SllmError):
        op.embedding(x, torch.zeros(4, dtype=torch.int64, device="cuda"), out=x)
    with pytest.raises(ValueError):
        op.embedding(x, torch.zeros(8, dtype=torch.int64, device="cuda")[::2])
    L = binding.lib()
    dst = torch.empty(64, dtype=torch.uint8)
    code = L.sllm_mx_quantize(binding.Matrix(dst.data_ptr(), 1, 32, 32, 2, 0), w[:1]._struct, 0, None)
    assert code == -1  # shapes differ
    code = L.sllm_mx_quantize(binding.Matrix(dst.data_ptr(), 1, 96, 96, 2, 0), w[:1]._struct, 0, None)
    assert code == -1 and b"device memory" in L.sllm_last_error()
    # a matrix that runs past its allocation
    code = L.sllm_mx_quantize(binding.Matrix(x.data_ptr(), 1 << 30, 96, 96, 2, 0),
                              binding.Mx(w.codes.data_ptr(), w.scales.data_ptr(), 1 << 30, 96), 0, None)
    assert code < 0
    # a workspace that is too small
    big = normal((200, 4096), torch.float16, 1)
    wide, _ = random_mx4(64, 4096, 1)
    y = torch.empty(200, 64, dtype=torch.float16, device="cuda")
    import ctypes as C

    n = C.c_uint64()
    args = (op._matrix(big, "x"), wide._struct)
    binding.check(L.sllm_mx_linear_workspace(*args, n))
    if n.value:
        assert L.sllm_mx_linear(*args, op._matrix(y, "y"), None, n.value - 1, 0, None) == -6
        assert L.sllm_mx_linear(*args, op._matrix(y, "y"), None, n.value, 0, None) == -1


def test_offsets_past_32_bits():
    """A table of more than 2^32 elements, looked up, quantised and its last rows used."""
    rows, cols = (1 << 32) // 4096 + 40, 4096
    table = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    table[-3:] = normal((3, cols), torch.bfloat16, 1)
    ids = torch.tensor([rows - 1, 0, rows - 3, rows], device="cuda")
    want = O.embedding(host(table[-3:]), [2, -1, 0, -1], 1.0)
    assert (host(op.embedding(table, ids)) == want).all()
    q = op.mx4_quantize(table)
    codes, scales = O.quantize(host(table[-3:]))
    assert (q.codes[-3:].cpu().numpy() == codes).all() and (q.scales[-3:].cpu().numpy() == scales).all()
    assert not q.codes[:-3].any()
    tail = O.dequantize(codes, scales, cols)
    assert (host(op.embedding(q, ids)) == O.embedding(tail, [2, -1, 0, -1], 1.0)).all()
    del table
    x = normal((2, cols), torch.bfloat16, 3)
    y = op.mx4_linear(x, q)
    assert_close(y[:, -3:], O.linear(host(x), tail), sum_bound(host(x), tail.T, cols), torch.bfloat16)
    assert not y[:, :-3].any()
    dy = torch.zeros(2, rows, dtype=torch.bfloat16, device="cuda")
    dy[:, -3:] = normal((2, 3), torch.bfloat16, 4)
    dx = op.mx4_linear_grad(dy, q)
    a = host(dy[:, -3:])
    assert_close(dx, O.linear_grad(a, tail), sum_bound(a, tail, rows), torch.bfloat16)
    grad = op.embedding_grad(x, torch.tensor([rows - 2, 5], device="cuda"), rows)
    assert torch.equal(grad[rows - 2], x[0]) and torch.equal(grad[5], x[1])
    assert not grad[6:rows - 2].any() and not grad[:5].any() and not grad[-1].any()


@pytest.mark.parametrize("n", [1, 1000, 1024, 1025, 5000, 20000])
def test_embedding_grad_of_a_very_tall_table(n):
    """Tables of 2^22 rows and more sort by wider keys; just below that, by the narrow ones."""
    for vocab in ((1 << 22) - 2, (1 << 22) - 1, 1 << 22, (1 << 22) + 7):
        dy = normal((n, 8), torch.float32, n)
        g = gen(vocab)
        ids = torch.randint(vocab - 50, vocab + 2, (n,), generator=g, device="cuda")
        grad = op.embedding_grad(dy, ids, vocab)
        want = O.embedding_grad(host(dy), (ids - (vocab - 60)).tolist(), 60, 1.0)
        size = O.embedding_grad(np.abs(host(dy)), (ids - (vocab - 60)).tolist(), 60, 1.0)
        assert_close(grad[-60:], want, 2 * (n + 8) * 2.0 ** -24 * size, torch.float32)
        assert not grad[:-60].any()
