"""An Mx4 is its two tensors: what it hands to the operators follows them."""

import copy
import pickle

import pytest

torch = pytest.importorskip("torch")
from paper_2401_14351_amd import operators as op  # noqa: E402


@pytest.fixture
def q():
    g = torch.Generator().manual_seed(1)
    return op.Mx4(torch.randint(256, (5, 32), generator=g, dtype=torch.uint8),
                  torch.randint(256, (5, 16), generator=g, dtype=torch.uint8), 40)


def address(q):
    s = q._struct
    return s.codes, s.scales, s.rows, s.cols


def test_its_parts_are_not_exchanged(q):
    for name, value in (("codes", q.codes.clone()), ("scales", q.scales.clone()), ("rows", 4), ("cols", 33), ("other", 1)):
        with pytest.raises(AttributeError):
            setattr(q, name, value)
    assert address(q) == (q.codes.data_ptr(), q.scales.data_ptr(), 5, 40)
    assert (q.rows, q.cols, q.shape, q.nbytes) == (5, 40, (5, 40), 5 * 48)


def test_storage_that_was_exchanged_is_followed(q):
    codes, scales = q.codes.clone(), q.scales.clone()
    q.codes.data, q.scales.data = codes, scales
    assert address(q) == (codes.data_ptr(), scales.data_ptr(), 5, 40)
    q.codes.set_(torch.zeros(7, 32, dtype=torch.uint8))
    with pytest.raises(ValueError):  # the scales are of five rows
        q._struct
    q.scales.set_(torch.zeros(7, 16, dtype=torch.uint8))
    assert address(q)[2] == q.rows == 7
    q.codes.resize_(7, 16)
    with pytest.raises(ValueError):
        q._struct


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, lambda q: pickle.loads(pickle.dumps(q))])
def test_copies(q, make):
    c = make(q)
    assert type(c) is op.Mx4 and c.cols == 40 and torch.equal(c.codes, q.codes) and torch.equal(c.scales, q.scales)
    assert address(c) == (c.codes.data_ptr(), c.scales.data_ptr(), 5, 40)
    assert (c.codes.data_ptr() == q.codes.data_ptr()) == (make is copy.copy)


def test_a_module_with_a_weight_is_copied(q):
    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.w = q

    layer = Layer()
    other = copy.deepcopy(layer)
    assert other.w is not q and torch.equal(other.w.codes, q.codes)
    q.codes.zero_()
    assert other.w.codes.any()
