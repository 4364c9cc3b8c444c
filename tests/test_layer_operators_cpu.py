"""The oracle of norms and attention against differences and hand-worked values, the
structs against the header, and what the entry points refuse before any device work."""

import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

from oracle import layer_oracle as O
from paper_2401_14351_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libsllm.so not built")
    return binding.lib()


# ---- the oracle -------------------------------------------------------------

def test_e4m3():
    assert len(O.E4M3) == 127 and O.E4M3[-1] == 448 and O.E4M3[1] == 2.0 ** -9 and O.E4M3[8] == 2.0 ** -6
    x = np.zeros((1, 32))
    x[0, :9] = [448, 17, 19, 18, -2.0 ** -10, 1.5 * 2.0 ** -9, 0, -0.0, 2.0 ** -11]
    codes, scales = O.quantize8(x)
    assert scales[0, 0] == 127
    assert O.dequantize8(codes, scales, 32)[0, :9].tolist() == [448, 16, 20, 18, 0, 2 * 2.0 ** -9, 0, 0, 0]
    assert codes[0, 4] == 0x80 and codes[0, 7] == 0x80


@pytest.mark.parametrize("top,scale", [(448.0, 127), (448.5, 128), (449.0, 128), (256.0, 127), (1.0, 119), (1.75, 119), (1.76, 120),
                                       (2.0 ** -119, 0), (2.0 ** -140, 0), (0.0, 0), (3e38, 247)])
def test_scales8(top, scale):
    x = np.zeros((1, 32))
    x[0, 5] = top
    assert O.quantize8(x)[1][0, 0] == scale


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_block_that_is_not_finite_is_nan(bad):
    x = np.ones((1, 64))
    x[0, 3] = bad
    codes, scales = O.quantize8(x)
    assert scales[0, :2].tolist() == [255, 119] and not codes[0, :32].any()
    v = O.dequantize8(codes, scales, 64)[0]
    assert np.isnan(v[:32]).all() and (v[32:] == 1).all()


def difference(f, x, at, step=1e-5):
    d = np.zeros_like(x)
    d[at] = step
    return (f(x + d) - f(x - d)) / (2 * step)


def test_norm_gradients_are_differences():
    rng = np.random.default_rng(0)
    h, gain, dy, dh = rng.normal(size=(3, 5)), rng.normal(size=5), rng.normal(size=(3, 5)), rng.normal(size=(3, 5))
    dx, dgain = O.norm_grad(dy, dh, h, gain, 1e-3)
    for i in range(3):
        for j in range(5):
            assert abs(difference(lambda x: (O.norm(x, gain, 1e-3) * dy + x * dh).sum(), h, (i, j)) - dx[i, j]) < 1e-8
    for j in range(5):
        assert abs(difference(lambda g: (O.norm(h, g, 1e-3) * dy).sum(), gain, (j,)) - dgain[j]) < 1e-8


@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (3, 0), (2, 1), (3, 4)])
def test_attention_gradients_are_differences(window, sinks):
    rng = np.random.default_rng(1)
    n, d = 7, 3
    q, k, v, dout = (rng.normal(size=(n, d)) for _ in range(4))
    seen = O.visible(range(n), range(n), window, sinks)
    assert (seen.sum(1) >= 1).all()
    grads = O.attend_grad(dout, q, k, v, seen, 0.7)
    for which, g in enumerate(grads):
        for i in range(n):
            for j in range(d):
                def f(x):
                    args = [q, k, v]
                    args[which] = x
                    return (O.attend(*args, seen, 0.7)[0] * dout).sum()
                assert abs(difference(f, (q, k, v)[which], (i, j)) - g[i, j]) < 1e-8


def test_who_sees_whom():
    assert O.visible([5], range(8), 3, 2)[0].tolist() == [True, True, False, True, True, True, False, False]
    assert O.visible([5], range(8), None, 0)[0].tolist() == [True] * 6 + [False] * 2
    assert [O.slot(p, 3, 2) for p in range(9)] == [0, 1, 2, 3, 4, 2, 3, 4, 2]


# ---- the boundary -----------------------------------------------------------

def test_struct_layouts_match_header(tmp_path):
    structs = {"sllm_heads": binding.Heads, "sllm_kv_cache": binding.KvCache}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sllm.h"', "int main(void) {"]
    for name, py in structs.items():
        lines.append(f'printf("{name} %zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in py._fields_]
        lines.append('printf("\\n");')
    (tmp_path / "p.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", f"-I{os.path.join(ROOT, 'include')}", str(tmp_path / "p.c"), "-o", str(tmp_path / "p")], check=True)
    out = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True).stdout.split("\n")
    for line, (name, py) in zip(out, structs.items()):
        assert line == f"{name} " + " ".join(map(str, [C.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]))


P = 1 << 24  # addresses that are never read: the calls below fail before device work
F32, BF16, I8 = 0, 2, 3
INVAL, RANGE = -1, -6
BIG = 1 << 31


def matrix(rows=4, cols=64, data=P, stride=None, dtype=BF16, reserved=0):
    return binding.Matrix(data, rows, cols, cols if stride is None else stride, dtype, reserved)


def mx(rows=8, cols=64, codes=2 * P, scales=3 * P):
    return binding.Mx(codes, scales, rows, cols)


def heads(tokens=4, n=8, dim=64, data=P, token_stride=None, head_stride=None, dtype=BF16, reserved=0):
    return binding.Heads(data, tokens, n, dim, n * dim if token_stride is None else token_stride, dim if head_stride is None else head_stride,
                         dtype, reserved)


def cache(sequences=4, n=2, dim=64, window=8, sinks=2, k=20 * P, v=21 * P, dtype=BF16, reserved=0):
    return binding.KvCache(k, v, sequences, n, dim, window, sinks, dtype, reserved)


def ids(n=5, data=4 * P, bits=32, reserved=0):
    return binding.Ids(data, n, bits, reserved)


Q, K, V, OUT = heads(), heads(n=2, data=2 * P), heads(n=2, data=3 * P), heads(data=5 * P)
S = C.c_float(0.125)


def attention(q=Q, k=K, v=V, offsets=None, window=0, sinks=0, scale=S, out=OUT, lse=None):
    return q, k, v, offsets, window, sinks, scale, out, lse, 0, None


def cached(q=Q, k=K, v=V, c=cache(), lengths=ids(4, 6 * P), offsets=ids(5, 7 * P), scale=S, out=OUT, ws=None, n=0):
    return q, k, v, c, lengths, offsets, scale, out, ws, n, 0, None


def attention_grad(dout=heads(data=8 * P), q=Q, k=K, v=V, out=OUT, lse=9 * P, offsets=None, scale=S, dq=heads(data=10 * P),
                   dk=heads(n=2, data=11 * P), dv=heads(n=2, data=12 * P), ws=13 * P, n=1 << 30):
    return dout, q, k, v, out, lse, offsets, 0, 0, scale, dq, dk, dv, ws, n, 0, None


def norm(x=matrix(), residual=None, gain=matrix(1, data=3 * P, dtype=F32), eps=1e-5, h=None, y=matrix(data=2 * P), inverse=None):
    return x, residual, gain, eps, h, y, inverse, 0, None


def norm_grad(dy=matrix(), dh=None, h=matrix(data=2 * P), gain=matrix(1, data=3 * P, dtype=F32), inverse=4 * P, dx=matrix(data=5 * P),
              dgain=matrix(1, data=6 * P, dtype=F32), ws=7 * P, n=1 << 20):
    return dy, dh, h, gain, inverse, dx, dgain, ws, n, 0, None


REFUSED = [
    ("sllm_attention", attention(q=None), INVAL),
    ("sllm_attention", attention(k=None), INVAL),
    ("sllm_attention", attention(v=None), INVAL),
    ("sllm_attention", attention(out=None), INVAL),
    ("sllm_attention", attention(q=heads(dtype=I8)), INVAL),
    ("sllm_attention", attention(q=heads(dtype=F32)), INVAL),
    ("sllm_attention", attention(q=heads(reserved=1)), INVAL),
    ("sllm_attention", attention(q=heads(data=P + 1)), INVAL),
    ("sllm_attention", attention(q=heads(data=None)), INVAL),
    ("sllm_attention", attention(q=heads(n=7)), INVAL),
    ("sllm_attention", attention(q=heads(n=3), out=heads(n=3, data=5 * P)), INVAL),       # 3 heads over 2
    ("sllm_attention", attention(k=heads(n=0, data=2 * P), v=heads(n=0, data=3 * P)), INVAL),
    ("sllm_attention", attention(k=heads(tokens=5, n=2, data=2 * P)), INVAL),
    ("sllm_attention", attention(v=heads(n=4, data=3 * P)), INVAL),
    ("sllm_attention", attention(v=heads(n=2, dim=32, data=3 * P)), INVAL),
    ("sllm_attention", attention(out=heads(dtype=F32, data=5 * P)), INVAL),
    ("sllm_attention", attention(out=heads(tokens=3, data=5 * P)), INVAL),
    ("sllm_attention", attention(out=heads(token_stride=511, data=5 * P)), INVAL),        # tokens overlap
    ("sllm_attention", attention(out=heads(head_stride=63, data=5 * P)), INVAL),
    ("sllm_attention", attention(q=heads(token_stride=0)), INVAL),
    ("sllm_attention", attention(q=heads(dim=129), k=heads(n=2, dim=129), v=heads(n=2, dim=129)), RANGE),
    ("sllm_attention", attention(q=heads(tokens=1 << 28)), RANGE),
    ("sllm_attention", attention(q=heads(token_stride=1 << 62)), RANGE),
    ("sllm_attention", attention(offsets=ids(0)), INVAL),
    ("sllm_attention", attention(offsets=ids(bits=16)), INVAL),
    ("sllm_attention", attention(offsets=ids(data=4 * P + 2)), INVAL),
    ("sllm_attention", attention(offsets=ids(1 << 24)), RANGE),
    ("sllm_attention", attention(scale=C.c_float(0)), INVAL),
    ("sllm_attention", attention(scale=C.c_float(-1)), INVAL),
    ("sllm_attention", attention(scale=C.c_float(math.inf)), INVAL),
    ("sllm_attention", attention(scale=C.c_float(math.nan)), INVAL),
    ("sllm_attention", attention(lse=5), INVAL),
    ("sllm_attention", attention(out=heads(data=P + 64)), INVAL),                         # overlaps q
    ("sllm_attention", attention(offsets=ids(data=5 * P)), INVAL),                        # overlaps out
    ("sllm_attention_cached", cached(c=None), INVAL),
    ("sllm_attention_cached", cached(lengths=None), INVAL),
    ("sllm_attention_cached", cached(c=cache(window=0)), INVAL),
    ("sllm_attention_cached", cached(c=cache(reserved=1)), INVAL),
    ("sllm_attention_cached", cached(c=cache(dtype=F32)), INVAL),
    ("sllm_attention_cached", cached(c=cache(n=4)), INVAL),
    ("sllm_attention_cached", cached(c=cache(dim=32)), INVAL),
    ("sllm_attention_cached", cached(c=cache(sequences=3)), INVAL),
    ("sllm_attention_cached", cached(c=cache(k=None)), INVAL),
    ("sllm_attention_cached", cached(c=cache(k=20 * P + 1)), INVAL),
    ("sllm_attention_cached", cached(c=cache(v=20 * P)), INVAL),                          # k and v overlap
    ("sllm_attention_cached", cached(c=cache(k=P)), INVAL),                               # overlaps q
    ("sllm_attention_cached", cached(c=cache(window=1 << 30, sinks=1)), RANGE),
    ("sllm_attention_cached", cached(c=cache(sinks=1 << 62)), RANGE),
    ("sllm_attention_cached", cached(lengths=ids(5, 6 * P)), INVAL),
    ("sllm_attention_cached", cached(offsets=ids(4, 7 * P)), INVAL),
    ("sllm_attention_cached", cached(offsets=None, c=cache(sequences=5), lengths=ids(5, 6 * P)), INVAL),
    ("sllm_attention_cached", cached(offsets=None, c=cache(window=1 << 20)), RANGE),      # no workspace
    ("sllm_attention_cached", cached(lengths=ids(4, 20 * P)), INVAL),                     # lengths in the cache
    ("sllm_attention_cached_workspace", (Q, K, V, cache(), ids(4), None, None), INVAL),
    ("sllm_attention_cached_workspace", (Q, K, V, cache(), ids(3), None, C.c_uint64()), INVAL),
    ("sllm_attention_grad", attention_grad(dout=None), INVAL),
    ("sllm_attention_grad", attention_grad(dout=heads(tokens=3, data=8 * P)), INVAL),
    ("sllm_attention_grad", attention_grad(lse=None), INVAL),
    ("sllm_attention_grad", attention_grad(out=None), INVAL),
    ("sllm_attention_grad", attention_grad(dq=None), INVAL),
    ("sllm_attention_grad", attention_grad(dk=heads(data=11 * P)), INVAL),
    ("sllm_attention_grad", attention_grad(dv=None), INVAL),
    ("sllm_attention_grad", attention_grad(dv=heads(n=2, data=11 * P)), INVAL),           # dk and dv overlap
    ("sllm_attention_grad", attention_grad(n=8), RANGE),
    ("sllm_attention_grad", attention_grad(ws=13 * P + 4), INVAL),
    ("sllm_attention_grad_workspace", (Q, K, None, 0, 0, None), INVAL),
    ("sllm_attention_grad_workspace", (Q, heads(n=3), None, 0, 0, C.c_uint64()), INVAL),
    ("sllm_rms_norm", norm(x=None), INVAL),
    ("sllm_rms_norm", norm(y=None), INVAL),
    ("sllm_rms_norm", norm(gain=None), INVAL),
    ("sllm_rms_norm", norm(gain=matrix(2, data=3 * P)), INVAL),
    ("sllm_rms_norm", norm(gain=matrix(1, 63, data=3 * P)), INVAL),
    ("sllm_rms_norm", norm(y=matrix(3, data=2 * P)), INVAL),
    ("sllm_rms_norm", norm(y=matrix(data=2 * P, dtype=F32)), INVAL),
    ("sllm_rms_norm", norm(residual=matrix(data=8 * P)), INVAL),                          # no h
    ("sllm_rms_norm", norm(h=matrix(data=8 * P)), INVAL),                                 # no residual
    ("sllm_rms_norm", norm(residual=matrix(5, data=8 * P), h=matrix(data=9 * P)), INVAL),
    ("sllm_rms_norm", norm(residual=matrix(data=8 * P, dtype=F32), h=matrix(data=9 * P)), INVAL),
    ("sllm_rms_norm", norm(residual=matrix(data=8 * P), h=matrix(data=2 * P)), INVAL),    # h and y overlap
    ("sllm_rms_norm", norm(y=matrix(data=P)), INVAL),
    ("sllm_rms_norm", norm(eps=-1.0), INVAL),
    ("sllm_rms_norm", norm(eps=math.nan), INVAL),
    ("sllm_rms_norm", norm(inverse=3), INVAL),
    ("sllm_rms_norm", norm(x=matrix(BIG)), RANGE),
    ("sllm_rms_norm_octet", (matrix(8), None, matrix(1), 1e-5, None, None, 0, None), INVAL),
    ("sllm_rms_norm_octet", (matrix(8), None, matrix(1), 1e-5, None, mx(7), 0, None), INVAL),
    ("sllm_rms_norm_octet", (matrix(8), None, matrix(1), 1e-5, None, mx(codes=2 * P + 8), 0, None), INVAL),
    ("sllm_rms_norm_grad", norm_grad(dy=None), INVAL),
    ("sllm_rms_norm_grad", norm_grad(h=matrix(3, data=2 * P)), INVAL),
    ("sllm_rms_norm_grad", norm_grad(dh=matrix(data=8 * P, dtype=F32)), INVAL),
    ("sllm_rms_norm_grad", norm_grad(inverse=None), INVAL),
    ("sllm_rms_norm_grad", norm_grad(dgain=matrix(1, data=6 * P)), INVAL),                # not gain's dtype
    ("sllm_rms_norm_grad", norm_grad(dx=None), INVAL),
    ("sllm_rms_norm_grad", norm_grad(n=16), RANGE),
    ("sllm_rms_norm_grad_workspace", (4, 64, None), INVAL),
    ("sllm_rms_norm_grad_workspace", (BIG, 64, C.c_uint64()), RANGE),
    ("sllm_mx_octet_sizes", (1, 1, None, None), INVAL),
    ("sllm_mx_octet_sizes", (BIG, 1, C.c_uint64(), C.c_uint64()), RANGE),
    ("sllm_mx_octet_quantize", (None, mx(), 0, None), INVAL),
    ("sllm_mx_octet_quantize", (matrix(7), mx(), 0, None), INVAL),
    ("sllm_mx_octet_quantize", (matrix(8), mx(codes=P), 0, None), INVAL),
    ("sllm_mx_octet_dequantize", (mx(), matrix(8, 65), 0, None), INVAL),
    ("sllm_mx_linear_octet", (None, mx(), matrix(4, 8), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_octet", (mx(4, 96), mx(), matrix(4, 8), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_octet", (mx(4), mx(codes=5 * P, scales=6 * P), matrix(4, 9, data=7 * P), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_octet", (mx(4), mx(codes=5 * P, scales=6 * P), matrix(4, 8, data=7 * P, dtype=F32), None, 0, 0, None), RANGE),
    ("sllm_mx_linear_octet_workspace", (mx(4), mx(), I8, C.c_uint64()), INVAL),
    ("sllm_mx_linear_octet_workspace", (mx(4), mx(), BF16, None), INVAL),
]


@pytest.mark.parametrize("i", range(len(REFUSED)), ids=lambda i: f"{i}-{REFUSED[i][0][5:]}")
def test_refused_arguments(L, i):
    name, args, code = REFUSED[i]
    assert getattr(L, name)(*args) == code, L.sllm_last_error()
    assert L.sllm_last_error()


@pytest.mark.parametrize("tokens,n,kv,dim", [(0, 0, 0, 0), (0, 8, 2, 64), (4, 8, 2, 0), (1, 1, 1, 1), (1 << 20, 64, 8, 128)])
def test_workspaces_of_any_shape(L, tokens, n, kv, dim):
    """Host-only, so empty operands are answered here too."""
    size = C.c_uint64()
    for dtype in (0, 1, 2):
        q, k = heads(tokens, n, dim, dtype=dtype), heads(tokens, kv, dim, dtype=dtype)
        for window, sinks in ((0, 0), (1, 1), (100, 1 << 40), (1 << 40, 4)):
            assert L.sllm_attention_grad_workspace(q, k, None, window, sinks, size) == 0
            assert L.sllm_attention_grad_workspace(q, k, ids(3), window, sinks, size) == 0
        if tokens <= 4096:
            c = cache(tokens, kv, dim, 4096, 4, dtype=dtype)
            assert L.sllm_attention_cached_workspace(q, k, k, c, ids(tokens), None, size) == 0
            assert L.sllm_attention_cached_workspace(q, k, k, c, ids(tokens), ids(tokens + 1), size) == 0 and size.value == 0
        assert L.sllm_rms_norm_grad_workspace(tokens, dim, size) == 0
        assert L.sllm_mx_linear_octet_workspace(mx(tokens, dim), mx(n, dim), dtype, size) == 0


def test_octet_sizes(L):
    a, b = C.c_uint64(), C.c_uint64()
    for rows, cols, codes, scales in ((0, 5, 0, 0), (1, 1, 32, 16), (5, 33, 320, 80), (7, 513, 7 * 544, 7 * 32)):
        binding.check(L.sllm_mx_octet_sizes(rows, cols, a, b))
        assert (a.value, b.value) == (codes, scales)


def test_python_refuses():
    torch = pytest.importorskip("torch")
    from paper_2401_14351_amd import operators as op

    x = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError):  # not in device memory
        op.attention(x, x, x)
    with pytest.raises(ValueError):
        op.rms_norm(torch.zeros(4, 8), torch.ones(8))
    with pytest.raises(ValueError):
        op.mx8_quantize(torch.zeros(4, 8))
    kv = torch.zeros(3, 2, 10, 8)
    c = op.KvCache(kv, kv.clone(), 8, 2)
    assert c[1:].k.data_ptr() == kv[1:].data_ptr() and c[1:].k.shape[0] == 2
    for args in ((kv, kv, 8, 1), (kv, kv, 0, 10), (kv, kv, 11, -1), (kv[:, :, ::2], kv[:, :, ::2], 5, 0), (kv, kv.half(), 8, 2),
                 (kv, kv[:2], 8, 2), (kv[0], kv[0], 8, 2), (kv.to(torch.int8), kv.to(torch.int8), 8, 2)):
        with pytest.raises(ValueError):
            op.KvCache(*args)
    for index in (0, slice(None, None, 2)):
        with pytest.raises(ValueError):
            c[index]
    with pytest.raises(ValueError):
        op.attention_cached(x[:3], x[:3], x[:3], c, None)
    u8 = torch.zeros(4, 64, dtype=torch.uint8)
    q = op.Mx8(u8, torch.zeros(4, 16, dtype=torch.uint8), 40)
    assert q.shape == (4, 40) and q[1:3].shape == (2, 40) and q.nbytes == 4 * 80 and "Mx8" in repr(q)
    with pytest.raises(ValueError):
        op.Mx8(u8[:, :32], torch.zeros(4, 16, dtype=torch.uint8), 40)
    with pytest.raises(ValueError):
        op.mx8_dequantize(op.Mx4(u8[:, :32].contiguous(), torch.zeros(4, 16, dtype=torch.uint8), 40))
    with pytest.raises(ValueError):
        q[1]


def test_python_refuses_what_requires_a_gradient():
    """Without a GPU too, whose streams it does not ask for."""
    torch = pytest.importorskip("torch")
    from paper_2401_14351_amd import operators as op

    x = torch.zeros(4, 2, 8, requires_grad=True)
    with pytest.raises(ValueError):
        op.attention(x, x, x)
    with pytest.raises(ValueError):
        op.rms_norm(x[0], torch.ones(8))


def test_grids_stay_within_what_can_be_launched(L):
    """Sequences, heads and both together, at their limits and one past them."""
    size = C.c_uint64()

    def grad(n, sequences):
        return L.sllm_attention_grad_workspace(heads(0, n), heads(0, n), ids(sequences + 1), 0, 0, size)

    def step(n, sequences):
        q = heads(sequences, n)
        return L.sllm_attention_cached_workspace(q, q, q, cache(sequences, n, window=1), ids(sequences), None, size)

    assert grad(64, 1 << 16) == 0 and grad(64, (1 << 16) + 1) == RANGE and grad(65, 1 << 16) == RANGE and grad(1, (1 << 16) + 1) == RANGE
    assert grad(1 << 16, 64) == 0 and grad((1 << 16) + 1, 1) == RANGE
    assert step(1, 1 << 22) == 0 and step(8, 1 << 19) == 0 and step(8, (1 << 19) + 1) == RANGE
