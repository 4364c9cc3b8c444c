"""The operators' oracle against hand-worked values, their structs against the
header, and the arguments the entry points refuse before any device work."""

import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

from oracle import operators_oracle as O
from paper_2401_14351_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libsllm.so not built")
    return binding.lib()


# ---- the oracle -------------------------------------------------------------

def block(*values):
    x = np.zeros((1, 32))
    x[0, :len(values)] = values
    return x


def test_levels_and_ties():
    # a largest magnitude in [4, 8) has scale 1
    x = block(6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 0.26, -0.74, -7.9, -0.0)
    codes, scales = O.quantize(x)
    assert scales[0, 0] == 127 and not scales[0, 1:].any()
    v = O.dequantize(codes, scales, 32)[0]
    assert v[:13].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 6, 0.5, -0.5, -6, 0]
    assert codes[0, 0] == 0x07 and codes[0, 6] >> 4 == 0  # 6 then 0.25; column 13 is zero
    assert codes[0, 6] & 15 == 8  # minus zero keeps its sign


@pytest.mark.parametrize("top,scale", [(1.0, 125), (1.99, 125), (2.0, 126), (0.02, 119), (2.0 ** -125, 0),
                                       (2.0 ** -149, 0), (0.0, 0), (3e38, 252)])
def test_scales(top, scale):
    assert O.quantize(block(top))[1][0, 0] == scale


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_block_that_is_not_finite_is_nan(bad):
    x = np.ones((1, 64))
    x[0, 3] = bad
    codes, scales = O.quantize(x)
    assert scales[0, :2].tolist() == [255, 125] and not codes[0, :16].any()
    v = O.dequantize(codes, scales, 64)[0]
    assert np.isnan(v[:32]).all() and (v[32:] == 1).all()


def test_values_of_the_format_come_back():
    rng = np.random.default_rng(0)
    x = rng.choice(O.LEVELS, (7, 50)) * rng.choice([-1, 1], (7, 50)) * 2.0 ** -6
    x[:, ::32] = 6 * 2.0 ** -6  # so that every block has this scale
    codes, scales = O.quantize(x)
    assert codes.shape == (7, 32) and scales.shape == (7, 16)
    assert (O.dequantize(codes, scales, 50) == x).all()


def test_gradients_are_differences():
    rng = np.random.default_rng(1)
    x, w, dy = rng.normal(size=(3, 5)), rng.normal(size=(4, 5)), rng.normal(size=(3, 4))
    dx = O.linear_grad(dy, w)
    for i in range(3):
        for j in range(5):
            step = np.zeros_like(x)
            step[i, j] = 1e-4
            diff = ((O.linear(x + step, w) - O.linear(x - step, w)) * dy).sum() / 2e-4
            assert abs(diff - dx[i, j]) < 1e-9
    table, ids = rng.normal(size=(4, 2)), [1, 3, 1, -1, 7]
    dy = rng.normal(size=(5, 2))
    g = O.embedding_grad(dy, ids, 4, 0.5)
    for v in range(4):
        for c in range(2):
            step = np.zeros_like(table)
            step[v, c] = 1e-4
            diff = ((O.embedding(table + step, ids, 0.5) - O.embedding(table - step, ids, 0.5)) * dy).sum() / 2e-4
            assert abs(diff - g[v, c]) < 1e-9


# ---- the boundary -----------------------------------------------------------

def test_struct_layouts_match_header(tmp_path):
    structs = {"sllm_matrix": binding.Matrix, "sllm_mx": binding.Mx, "sllm_ids": binding.Ids}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sllm.h"', "int main(void) {"]
    for name, py in structs.items():
        lines.append(f'printf("{name} %zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in py._fields_]
        lines.append('printf("\\n");')
    (tmp_path / "p.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", f"-I{os.path.join(ROOT, 'include')}", str(tmp_path / "p.c"), "-o", str(tmp_path / "p")],
                   check=True)
    out = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True).stdout.split("\n")
    for line, (name, py) in zip(out, structs.items()):
        want = [C.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]
        assert line == f"{name} " + " ".join(map(str, want))


@pytest.mark.parametrize("rows,cols,codes,scales", [(0, 5, 0, 0), (3, 0, 0, 0), (1, 1, 16, 16), (2, 32, 32, 32),
                                                    (5, 33, 160, 80), (7, 512, 7 * 256, 7 * 16),
                                                    (7, 513, 7 * 272, 7 * 32), (1 << 30, 1 << 20, 1 << 49, 1 << 45)])
def test_sizes(L, rows, cols, codes, scales):
    a, b = C.c_uint64(), C.c_uint64()
    binding.check(L.sllm_mx_sizes(rows, cols, a, b))
    assert (a.value, b.value) == (codes, scales)


P = 1 << 20  # addresses that are never read: the calls below fail before device work
BF16, I8 = 2, 3


def matrix(rows=4, cols=64, data=P, stride=None, dtype=BF16, reserved=0):
    return binding.Matrix(data, rows, cols, cols if stride is None else stride, dtype, reserved)


def mx(rows=8, cols=64, codes=2 * P, scales=3 * P):
    return binding.Mx(codes, scales, rows, cols)


def ids(n=4, data=4 * P, bits=32, reserved=0):
    return binding.Ids(data, n, bits, reserved)


def out(rows=4, cols=8, data=5 * P, **kw):
    return matrix(rows, cols, data, **kw)


INVAL, RANGE = -1, -6
BIG = 1 << 31


@pytest.mark.parametrize("name,args,code", [
    ("sllm_mx_sizes", (1, 1, None, None), INVAL),
    ("sllm_mx_sizes", (BIG, 1, C.c_uint64(), C.c_uint64()), RANGE),
    ("sllm_mx_quantize", (None, mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8), None, 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(7), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8, dtype=I8), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8, reserved=1), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8, data=P + 1), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8, data=None), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8, stride=63), mx(), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8), mx(codes=2 * P + 8), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8), mx(scales=3 * P + 8), 0, None), INVAL),
    ("sllm_mx_quantize", (matrix(8), mx(scales=None), 0, None), INVAL),
    ("sllm_mx_dequantize", (mx(), matrix(8, 65), 0, None), INVAL),
    ("sllm_mx_dequantize", (mx(BIG), matrix(BIG), 0, None), RANGE),
    ("sllm_mx_dequantize", (mx(), matrix(8, stride=1 << 62), 0, None), RANGE),
    ("sllm_mx_linear", (None, mx(), out(), None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(), None, out(), None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(), mx(), None, None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(cols=63), mx(), out(), None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(), mx(), out(cols=9), None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(), mx(), out(rows=5), None, 0, 0, None), INVAL),
    ("sllm_mx_linear", (matrix(), mx(), out(stride=7), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_mx", (None, mx(), out(), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_mx", (mx(4, 96), mx(), out(), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_grad", (matrix(cols=9), mx(), out(cols=64), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_grad", (None, mx(), out(cols=64), None, 0, 0, None), INVAL),
    ("sllm_mx_linear_workspace", (matrix(), mx(), None), INVAL),
    ("sllm_mx_linear_workspace", (None, mx(), C.c_uint64()), INVAL),
    ("sllm_mx_linear_mx_workspace", (mx(4, 32), mx(), C.c_uint64()), INVAL),
    ("sllm_mx_linear_grad_workspace", (matrix(), mx(), C.c_uint64()), INVAL),
    ("sllm_embedding", (None, ids(), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding", (matrix(), None, 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding", (matrix(), ids(bits=16), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding", (matrix(), ids(reserved=1), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding", (matrix(), ids(data=4 * P + 4, bits=64), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding", (matrix(), ids(), 1.0, out(cols=63), 0, None), INVAL),
    ("sllm_embedding", (matrix(), ids(5), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding_mx", (None, ids(), 1.0, out(cols=64), 0, None), INVAL),
    ("sllm_embedding_mx", (mx(), ids(), 1.0, out(cols=65), 0, None), INVAL),
    ("sllm_embedding_grad", (matrix(), ids(), 1.0, 2, out(cols=64), P, 1 << 40, 0, None), INVAL),
    ("sllm_embedding_grad", (matrix(), ids(3), 1.0, 0, out(cols=64), P, 1 << 40, 0, None), INVAL),
    ("sllm_embedding_grad", (matrix(), ids(), 1.0, 0, out(cols=63), P, 1 << 40, 0, None), INVAL),
    ("sllm_embedding_grad", (matrix((1 << 24) + 1), ids((1 << 24) + 1), 1.0, 0, out(cols=64), P, 1 << 40, 0, None), RANGE),
    ("sllm_embedding_grad_workspace", ((1 << 24) + 1, out(cols=64), C.c_uint64()), RANGE),
    ("sllm_embedding_grad_workspace", (4, None, C.c_uint64()), INVAL),
])
def test_refused_arguments(L, name, args, code):
    assert getattr(L, name)(*args) == code
    assert L.sllm_last_error()


def test_python_refuses():
    torch = pytest.importorskip("torch")
    from paper_2401_14351_amd import operators as op

    u8 = torch.zeros(4, 32, dtype=torch.uint8)
    q = op.Mx4(u8, torch.zeros(4, 16, dtype=torch.uint8), 40)
    assert q.shape == (4, 40) and q[1:3].shape == (2, 40) and q.nbytes == 4 * 48
    assert q[1:].codes.data_ptr() == u8.data_ptr() + 32
    for codes, scales, cols in ((u8, u8, 40), (u8, u8[:, :16], 40), (u8[:, ::2], u8[:, ::2], 16), (u8.int(), u8, 40),
                                (u8, torch.zeros(3, 16, dtype=torch.uint8), 40), (u8[0], u8[0], 40)):
        with pytest.raises(ValueError):
            op.Mx4(codes, scales, cols)
    with pytest.raises(ValueError):
        q[::2]
    with pytest.raises(ValueError):
        q[1]
    with pytest.raises(ValueError):  # not in device memory
        op.mx4_quantize(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        op.mx4_quantize(torch.zeros(4, 4, dtype=torch.int8))
    with pytest.raises(ValueError):
        op.embedding_grad(torch.zeros(4, 4), torch.zeros(3, dtype=torch.int64), 8)
    with pytest.raises(ValueError):
        op.embedding_grad(torch.zeros(3, 4), torch.zeros(3, dtype=torch.int64), 8, accumulate=True)
    with pytest.raises(ValueError):
        op.embedding(torch.zeros(4, 4), torch.zeros(3))


@pytest.mark.parametrize("m,n,k", [(0, 0, 0), (0, 8, 64), (4, 0, 64), (4, 8, 0), (1, 1, 1), (4096, 28672, 8192)])
def test_workspaces_of_any_shape(L, m, n, k):
    """Host-only, so empty operands are answered here too."""
    size = C.c_uint64()
    for dtype in (0, 1, 2):
        assert L.sllm_mx_linear_workspace(matrix(m, k, dtype=dtype), mx(n, k), size) == 0
        assert L.sllm_mx_linear_grad_workspace(matrix(m, n, dtype=dtype), mx(n, k), size) == 0
        assert L.sllm_embedding_grad_workspace(m, matrix(n, k, dtype=dtype), size) == 0
    assert L.sllm_mx_linear_mx_workspace(mx(m, k), mx(n, k), size) == 0
