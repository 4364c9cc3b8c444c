"""The operators on loaded weights at the edges of their formats, types and sizes.

Tolerances are those of ``test_gpu_operators``: a sum of `depth` products in 32
bits is off by at most `sum_bound`, and an output's rounding adds half a unit in
its last place.
"""

import math

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


def spread(shape, seed, low, high):
    """float16 values of random signs whose exponents lie in [low, high), subnormals among them."""
    rng = np.random.default_rng(seed)
    v = np.ldexp(rng.uniform(1, 2, shape), rng.integers(low, high, shape)) * rng.choice([-1, 1], shape)
    return torch.from_numpy(v.astype(np.float16)).cuda()


@pytest.mark.parametrize("depth", [32, 64, 200])
@pytest.mark.parametrize("m,n", [(40, 512), (130, 130), (130, 4200), (2600, 4200)])
@pytest.mark.parametrize("scales,exponents", [((96, 98), (-10, 0)), ((96, 104), (-10, 0)), ((100, 133), (-24, -10)),
                                              ((100, 133), (-24, 15)), ((114, 128), (-24, 15)), ((106, 107), (-24, 0))])
def test_linear_half_exponents_apart(depth, m, n, scales, exponents):
    """Sums over few and small products lose no more than 32 bits do: W or x of any size that float16 has."""
    w, wv = random_mx4(n, depth, depth, scales)
    x = spread((m, depth), m, *exponents)
    a = host(x)
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, depth), torch.float32)
    g, gv = random_mx4(depth, n, depth, scales)
    assert_close(op.mx4_linear_grad(x, g, out_dtype=torch.float32), O.linear_grad(a, gv), sum_bound(a, gv, depth), torch.float32)


@pytest.mark.parametrize("m,n", [(40, 512), (130, 130), (2600, 4200)])
def test_linear_half_normal_over_zero(m, n):
    """One normal element, over weights of zero; the rest subnormal over blocks far apart in size."""
    depth = 64
    w, _ = random_mx4(n, depth, 3, (100, 133))
    w.codes[:, 0] &= 0xf0  # column 0
    wv = values(w)
    x = spread((m, depth), 4, -24, -14)
    x[:, 0] = 1.0
    a = host(x)
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, depth), torch.float32)
    g, _ = random_mx4(depth, n, 5, (100, 133))
    g.codes[0] = 0
    gv = values(g)
    assert_close(op.mx4_linear_grad(x, g, out_dtype=torch.float32), O.linear_grad(a, gv), sum_bound(a, gv, depth), torch.float32)


@pytest.mark.parametrize("depth", [203, 1501, 4096])
@pytest.mark.parametrize("first", [0, 1, 8])
def test_linear_half_ranges_of_any_rows(depth, first):
    """Rows copied first, by a wave or a workgroup each, and rows that are not: their ranges are their own."""
    m, n = 70, 300
    w, _ = random_mx4(n, depth, 7, (118, 128))
    w.codes[:, 16:] = 0  # sums of 32 products, so that no bits are lost in larger ones
    wv = values(w)
    base = spread((m, depth + 16), 8, -24, -13)  # rows start on 16 bytes for one depth and two firsts
    base[::3] *= 2.0 ** 13
    base[1::3, first + 40] = 40000  # the smallest elements and a large one, over a weight of zero
    x = base[:, first:first + depth]
    a = host(x)
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a[:, :32], wv[:, :32].T, 32), torch.float32)
    g, _ = random_mx4(depth, n, 9, (118, 128))
    g.codes[32:] = 0
    gv = values(g)
    assert_close(op.mx4_linear_grad(x, g, out_dtype=torch.float32), O.linear_grad(a, gv), sum_bound(a[:, :32], gv[:32], 32),
                 torch.float32)


@pytest.mark.parametrize("m,n,k", ROWS)
def test_linear_half_outliers(m, n, k):
    """Elements up to float16's largest beside its smallest, a few of each."""
    w, wv = random_mx4(n, k, 6, (106, 133))
    for seed, part in ((1, 0.001), (2, 0.2)):
        def ragged(shape):
            rng = np.random.default_rng(seed)
            v = rng.normal(size=shape)
            v = np.where(rng.random(shape) < part, np.ldexp(v, rng.integers(5, 14, shape)), v)
            v = np.where(rng.random(shape) < part, np.ldexp(v, -rng.integers(10, 24, shape)), v)
            v.flat[0], v.flat[-1] = 65504, -64
            return torch.from_numpy(v.astype(np.float16)).cuda()

        x, dy = ragged((m, k)), ragged((m, n))
        a, b = host(x), host(dy)
        assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), sum_bound(a, wv.T, k), torch.float32)
        assert_close(op.mx4_linear_grad(dy, w, out_dtype=torch.float32), O.linear_grad(b, wv), sum_bound(b, wv, n), torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(1, 40), (4, 40), (16, 40), (40, 40), (300, 300)])
def test_linear_of_very_small_elements(dtype, m, n):
    """Elements below 2^-110 count to within 2^-133, which is bfloat16's smallest step; sums that are
    subnormal are off by half of float32's smallest step each."""
    depth = 96
    w, wv = random_mx4(n, depth, 8, (120, 150))
    rng = np.random.default_rng(9)
    v = np.ldexp(rng.uniform(1, 2, (m, depth)), rng.integers(-149, -100, (m, depth))) * rng.choice([-1, 1], (m, depth))
    x = torch.from_numpy(v.astype(np.float32)).cuda().to(dtype)
    a = host(x)
    small = np.full_like(a, 2.0 ** -133)
    bound = sum_bound(a, wv.T, depth) + small @ np.abs(wv).T + depth * 2.0 ** -149
    assert_close(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(a, wv), bound, torch.float32)
    g, gv = random_mx4(depth, n, 10, (120, 150))
    bound = sum_bound(a, gv, depth) + small @ np.abs(gv) + depth * 2.0 ** -149
    assert_close(op.mx4_linear_grad(x, g, out_dtype=torch.float32), O.linear_grad(a, gv), bound, torch.float32)


# ---- what is not finite -----------------------------------------------------

def assert_same_kind(got, want):
    """NaN and infinities, with their signs, where the definition has them."""
    g = host(got)
    assert (np.isnan(g) == np.isnan(want)).all()
    inf = np.isinf(want)
    assert (np.isinf(g) == inf).all() and (g[inf] == want[inf]).all()


def patterns(dtype):
    """A NaN whose payload is in its lowest bits alone, and others."""
    quiet = {torch.bfloat16: (0x7f81, torch.int16), torch.float16: (0x7c01, torch.int16), torch.float32: (0x7f800001, torch.int32)}
    bits, whole = quiet[dtype]
    low = torch.tensor([bits], dtype=whole).view(dtype)[0]
    return [torch.tensor(v, dtype=dtype) for v in (math.inf, -math.inf, math.nan)] + [low]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", ROWS)
@pytest.mark.parametrize("tiny_block", [False, True])
def test_not_finite_by_element(dtype, m, n, k, tiny_block):
    """An infinity of x over a zero weight is NaN, over others an infinity of its sign; a NaN is a NaN."""
    w, _ = random_mx4(n, k, 11, (118, 128))
    if tiny_block:  # a block that float16 does not hold
        w.scales[n // 2, 1] = 60
    wv = values(w)
    for i, bad in enumerate(patterns(dtype)):
        x, dy = normal((m, k), dtype, 12), normal((m, n), dtype, 13)
        x[m // 2, (i * 37 + 5) % k] = bad.cuda()
        dy[m - 1, n - 1 - i] = bad.cuda()
        with np.errstate(invalid="ignore"):
            assert_same_kind(op.mx4_linear(x, w, out_dtype=torch.float32), O.linear(host(x), wv))
            assert_same_kind(op.mx4_linear_grad(dy, w, out_dtype=torch.float32), O.linear_grad(host(dy), wv))


# ---- lookups ----------------------------------------------------------------

@pytest.mark.parametrize("scale", [-2.0, 0.0, -0.0, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [7, 96, 1100])
def test_padding_is_zeros_under_any_scale(scale, dtype, dim):
    table = normal((9, dim), dtype, 1)
    q = op.mx4_quantize(table)
    ids = torch.tensor([3, -1, 8, 9, 0, 1 << 40], device="cuda")
    for t in (table, q):
        y = op.embedding(t, ids, scale, out_dtype=dtype)
        for row in (1, 3, 5):
            assert not y[row].any() and not y[row].signbit().any()
        plain = (table if t is table else op.mx4_dequantize(q, torch.float32)).float()
        want = (plain[[3, 8, 0]] * scale).to(dtype)
        assert ((y[[0, 2, 4]] == want) | (y[[0, 2, 4]].isnan() & want.isnan())).all()


# ---- sizes ------------------------------------------------------------------

def test_more_rows_than_a_launch_of_one_dimension():
    """2^24 rows of more than 1024 columns: looked up, quantised and back."""
    rows, cols = (1 << 24) + 3, 1032
    table = normal((5, cols), torch.bfloat16, 1)
    ids = torch.zeros(rows, dtype=torch.int32, device="cuda")
    ids[-3:] = torch.tensor([4, 7, 2])
    y = op.embedding(table, ids)
    assert torch.equal(y[-3], table[4]) and not y[-2].any() and torch.equal(y[-1], table[2])
    assert torch.equal(y[(1 << 24) - 2:1 << 24], table[:1].expand(2, cols)) and torch.equal(y[0], table[0])
    q = op.mx4_quantize(y)
    few = op.mx4_quantize(y[-5:])
    assert torch.equal(q.codes[-5:], few.codes) and torch.equal(q.scales[-5:], few.scales)
    op.mx4_dequantize(q, out=y)
    assert torch.equal(y[-5:], op.mx4_dequantize(few)) and torch.equal(y[0], y[-5])


def test_gradient_of_a_table_of_many_rows():
    """More rows to clear than one dimension of a launch counts, 16 a workgroup."""
    vocab = (1 << 28) + 40
    out = torch.full((vocab, 1), 3.0, dtype=torch.float16, device="cuda")
    ids = torch.tensor([vocab - 1, 5, vocab - 2, 5, vocab], device="cuda")
    op.embedding_grad(torch.tensor([[1.0], [2.0], [4.0], [8.0], [16.0]], device="cuda"), ids, vocab, out=out)
    assert out[-1].item() == 1 and out[-2].item() == 4 and out[5].item() == 10
    out[-2:] = 0
    out[5] = 0
    assert not out.any()


def test_product_with_a_weight_of_many_rows():
    """2^30 rows of W and one of x: 2^26 workgroups."""
    n, k = (1 << 30) + 17, 32
    w = op.Mx4(torch.zeros(n, 16, dtype=torch.uint8, device="cuda"), torch.zeros(n, 16, dtype=torch.uint8, device="cuda"), k)
    small, sv = random_mx4(20, k, 1)
    w.codes[-20:], w.scales[-20:] = small.codes, small.scales
    x = normal((1, k), torch.bfloat16, 2)
    y = op.mx4_linear(x, w)
    a = host(x)
    assert_close(y[:, -20:], O.linear(a, sv), sum_bound(a, sv.T, k), torch.bfloat16)
    y[:, -20:] = 0
    assert not y.any()


# ---- tensors whose memory is not what they stand for ------------------------

def test_negated_views_are_refused():
    x = normal((4, 96), torch.float32, 1)
    w, _ = random_mx4(8, 96, 2)
    z = torch.complex(normal((4, 1), torch.float32, 3), normal((4, 1), torch.float32, 4)).conj().imag
    assert z.is_neg()
    thin, _ = random_mx4(8, 1, 5)
    neg = torch._neg_view(x)
    for call in (lambda: op.mx4_linear(neg, w), lambda: op.mx4_linear(z, thin), lambda: op.mx4_quantize(neg),
                 lambda: op.embedding(neg, torch.zeros(3, dtype=torch.int64, device="cuda")),
                 lambda: op.embedding(x, torch._neg_view(torch.zeros(3, dtype=torch.int64, device="cuda"))),
                 lambda: op.embedding_grad(neg, torch.zeros(4, dtype=torch.int64, device="cuda"), 3),
                 lambda: op.mx4_dequantize(w, out=torch._neg_view(normal((8, 96), torch.float32, 6)))):
        with pytest.raises(ValueError, match="negat"):
            call()


# ---- autograd ---------------------------------------------------------------

def test_a_changed_weight_raises_in_backward():
    w, wv = random_mx4(48, 64, 1)
    x = normal((9, 64), torch.float32, 2).requires_grad_()
    for change in (lambda: op.mx4_quantize(normal((48, 64), torch.float32, 3), out=w), lambda: w.scales.add_(1),
                   lambda: w.codes.zero_()):
        y = op.mx4_linear(x, w)
        change()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    w, wv = random_mx4(48, 64, 1)
    op.mx4_linear(x, w).sum().backward()
    assert_close(x.grad, O.linear_grad(np.ones((9, 48)), wv), sum_bound(np.ones((9, 48)), wv, 48), torch.float32)


@pytest.mark.parametrize("write", ["linear", "linear_mx", "linear_grad", "embedding", "embedding_grad", "accumulate", "dequantize"])
@pytest.mark.parametrize("stream", [False, True])
def test_a_written_output_raises_in_backward(write, stream):
    """A tensor saved for a backward pass and then written through out= is told from one that was not."""
    w, _ = random_mx4(32, 32, 1)
    x = normal((32, 32), torch.float32, 2)
    ids = torch.arange(32, device="cuda")
    held = torch.zeros(32, 32, device="cuda")
    keep = {"stream": torch.cuda.current_stream()} if stream else {}
    scale = torch.ones(32, 32, device="cuda", requires_grad=True)
    y = scale * held
    {"linear": lambda: op.mx4_linear(x, w, out=held, **keep),
     "linear_mx": lambda: op.mx4_linear(op.mx4_quantize(x), w, out=held, **keep),
     "linear_grad": lambda: op.mx4_linear_grad(x, w, out=held, **keep),
     "embedding": lambda: op.embedding(x, ids, out=held, **keep),
     "embedding_grad": lambda: op.embedding_grad(x, ids, 32, out=held, **keep),
     "accumulate": lambda: op.embedding_grad(x, ids, 32, out=held, accumulate=True, **keep),
     "dequantize": lambda: op.mx4_dequantize(w, out=held, **keep)}[write]()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_weights_of_inference_mode_serve_training():
    """They have no versions and cannot be saved, but their gradients are right."""
    with torch.inference_mode():
        w = op.mx4_quantize(normal((48, 64), torch.bfloat16, 1))
        out = torch.empty(48, 64, device="cuda")
        assert op.mx4_dequantize(w, out=out) is out
        op.mx4_quantize(normal((48, 64), torch.bfloat16, 1), out=w)
    wv = values(w)
    x = normal((9, 64), torch.float32, 2).requires_grad_()
    op.mx4_linear(x, w).sum().backward()
    assert_close(x.grad, O.linear_grad(np.ones((9, 48)), wv), sum_bound(np.ones((9, 48)), wv, 48), torch.float32)


def test_saved_weights_pass_the_hooks():
    w, wv = random_mx4(48, 64, 1)
    x = normal((9, 64), torch.float32, 2).requires_grad_()
    with torch.autograd.graph.save_on_cpu():
        y = op.mx4_linear(x, w)
    w.codes.zero_()  # what was saved is a copy
    y.sum().backward()
    assert_close(x.grad, O.linear_grad(np.ones((9, 48)), wv), sum_bound(np.ones((9, 48)), wv, 48), torch.float32)


def test_quantising_what_requires_a_gradient_is_refused():
    x = normal((9, 64), torch.float32, 1).requires_grad_()
    q = op.Mx4.empty(9, 64, "cuda")
    for call in (lambda: op.mx4_quantize(x), lambda: op.mx4_quantize(x, out=q), lambda: op.mx4_quantize(x * 2),
                 lambda: op.mx4_quantize(x, stream=torch.cuda.current_stream())):
        with pytest.raises(ValueError, match="gradient"):
            call()
    want = op.mx4_quantize(x.detach())
    with torch.no_grad():
        assert torch.equal(op.mx4_quantize(x).codes, want.codes)


def test_tangents_are_refused():
    import torch.autograd.forward_ad as forward

    w, _ = random_mx4(48, 64, 1)
    x, dy = normal((9, 64), torch.float32, 2), normal((9, 48), torch.float32, 3)
    ids = torch.arange(9, device="cuda")
    with forward.dual_level():
        a, b = forward.make_dual(x, torch.ones_like(x)), forward.make_dual(dy, torch.ones_like(dy))
        for call in (lambda: op.mx4_linear(a, w), lambda: op.mx4_linear_grad(b, w), lambda: op.embedding(a, ids),
                     lambda: op.embedding_grad(a, ids, 9), lambda: op.mx4_quantize(a),
                     lambda: op.mx4_linear(x, w, out=b), lambda: op.embedding(x, ids, out=a)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        plain = op.mx4_linear(x, w)  # others are carried out
    assert torch.equal(plain, op.mx4_linear(x, w))


def test_transformed_tensors_are_refused():
    """Tensors of torch.func's transforms have no memory of their own."""
    w, _ = random_mx4(48, 64, 1)
    x = normal((3, 9, 64), torch.float32, 2)
    for transform in (torch.vmap, lambda f: torch.func.grad(lambda x: f(x).sum()), lambda f: lambda x: torch.func.jvp(f, (x,), (x,))):
        with pytest.raises((RuntimeError, ValueError)):
            transform(lambda x: op.mx4_linear(x, w))(x)


# ---- weights that move ------------------------------------------------------

def test_storage_that_was_exchanged():
    """A weight is where its tensors are when it is used."""
    w, _ = random_mx4(48, 64, 1)
    v, vv = random_mx4(48, 64, 2)
    x = normal((20, 64), torch.bfloat16, 3)
    w.codes.data, w.scales.data = v.codes.clone(), v.scales.clone()
    a = host(x)
    assert_close(op.mx4_linear(x, w), O.linear(a, vv), sum_bound(a, vv.T, 64), torch.bfloat16)
    w.codes.data = v.codes[:40].clone()
    with pytest.raises(ValueError):
        op.mx4_linear(x, w)
