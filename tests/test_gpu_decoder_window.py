"""The decoder example over a window: a run of the operators as a decoder uses them."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    found = importlib.util.spec_from_file_location("mx4_decoder", os.path.join(ROOT, "examples", "mx4_decoder.py"))
    module = importlib.util.module_from_spec(found)
    found.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def views(example, tmp_path_factory):
    return example.load(example.checkpoint(3, 192, 200, 517, 1), str(tmp_path_factory.mktemp("decoder") / "ckpt"))


def text(n):
    return torch.randint(517, (n,), generator=torch.Generator().manual_seed(n)).cuda()


@pytest.mark.parametrize("window,sinks", [(7, 0), (16, 3), (1, 1), (None, 0)])
def test_pieces_give_the_logits_of_the_whole(example, views, window, sinks):
    """A text in pieces over the cache and at once over itself: in 32 bits, sums of up to 2000
    terms on the way to a logit are off by less than 2 * 2000 * 2^-24 < 2^-12 of the largest."""
    tokens = text(60)
    model = example.Decoder(views, torch.float32, window, sinks)
    with torch.no_grad():
        want = model.logits(tokens)
        cache, got, at = example.Cache(model), [], 0
        for n in (1, 20, 1, 1, 30, 1, 6):
            got.append(model.logits(tokens[at:at + n], cache))
            at += n
    assert (torch.cat(got) - want).abs().max() <= 2.0 ** -12 * want.abs().max()


def test_gradient_is_the_difference(example, views):
    """Along a direction, of the loss over a window with sinks; steps of 2^-6 leave about
    2^-12 of curvature and 2^-24 * 2^6 of rounding."""
    tokens = text(40)
    model = example.Decoder(views, torch.float32, 9, 2)
    table = model.table.clone().requires_grad_()

    def loss(t):
        return torch.nn.functional.cross_entropy(model.logits(tokens[:-1], table=t).double(), tokens[1:])

    loss(table).backward()
    along = torch.randn(table.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    along *= 2.0 ** -6 * model.table.std()
    with torch.no_grad():
        slope = (loss(table + along) - loss(table - along)) / 2
    got = (table.grad.double() * along).sum()
    scale = (table.grad.double().norm() * along.norm()).item()
    assert abs((got - slope).item()) <= 0.02 * scale


@pytest.mark.parametrize("bits", [None, 4, 8])
def test_answers(example, views, bits):
    model = example.Decoder(views, window=12, sinks=2)
    answer = model.answer(text(50), 8, bits=bits)
    assert answer.shape == (8,) and ((answer >= 0) & (answer < 517)).all()
    with torch.no_grad():
        assert torch.equal(model.logits(text(50), bits=bits), model.logits(text(50), bits=bits))


def test_eight_bits_are_near(example, views):
    """An element is off by at most 2^-4 of itself, about 2^-5.6 of it in root mean square; three
    layers of four products and the head's keep the logits within a third."""
    model = example.Decoder(views)
    with torch.no_grad():
        want, got = (model.logits(text(50), bits=b).double() for b in (None, 8))
    assert (got - want).norm() <= want.norm() / 3
