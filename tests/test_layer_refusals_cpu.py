"""More of what the layer's entry points refuse before any device work."""

import ctypes as C

import pytest

from tests.test_layer_operators_cpu import INVAL, L, attention, attention_grad, cached  # noqa: F401


@pytest.mark.parametrize("name,args", [("sllm_attention", attention), ("sllm_attention_cached", cached), ("sllm_attention_grad", attention_grad)])
def test_a_scale_whose_product_with_log2_e_leaves_32_bits(L, name, args):  # noqa: F811
    assert getattr(L, name)(*args(scale=C.c_float(3e38))) == INVAL
    assert b"scale" in L.sllm_last_error()
    assert getattr(L, name)(*args(scale=C.c_float(2.3e38), out=None)) == INVAL
    assert b"out" in L.sllm_last_error()  # the scale was taken
