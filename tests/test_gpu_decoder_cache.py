"""The decoder example's attention in 32 bits, over a cache."""

import pytest

from tests.test_gpu_decoder_window import example, text, views  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("window,sinks", [(None, 0), (9, 2)])
def test_attention_in_32_bits(example, views, window, sinks):  # noqa: F811
    """Of activations in 16 bits: rotated queries and keys and weights are not rounded to them, the result once.

    Sums of 64 and of 40 terms in 32 bits, their exponents below 16, angles below 40 radians: 2^-14 of the largest."""
    model = example.Decoder(views, torch.bfloat16, window, sinks)
    n, head = 40, example.HEAD
    qkv = torch.randn(n, model.dim + 2 * head, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(torch.bfloat16)
    with torch.no_grad():
        got = model.attention(qkv, None, 0).double().cpu()
    q, k, v = (t.unflatten(-1, (-1, head)).transpose(0, 1) for t in qkv.double().cpu().split([model.dim, head, head], -1))
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, head, 2, dtype=torch.float64) / head)

    def rotate(x):
        a, b = x[..., :head // 2], x[..., head // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    i, j = torch.arange(n)[:, None], torch.arange(n)
    seen = (j <= i) & ((i - j < (window or n)) | (j < sinks))
    s = (rotate(q) @ rotate(k).transpose(1, 2) * head ** -0.5).masked_fill(~seen, -float("inf"))
    want = (torch.softmax(s, -1) @ v).transpose(0, 1).flatten(1)
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -14 * want.abs().max()).all()


def test_a_cache_in_32_bits(example, views, monkeypatch):  # noqa: F811
    """And so is what is kept of a text whose activations have 16 bits."""
    seen = []

    def attention_cached(q, k, v, cache, *args, **kwargs):
        seen.extend(t.dtype for t in (q, k, v, cache.k, cache.v))
        return attend(q, k, v, cache, *args, **kwargs)

    attend = example.operators.attention_cached
    monkeypatch.setattr(example.operators, "attention_cached", attention_cached)
    model = example.Decoder(views, torch.bfloat16)
    assert len(model.answer(text(30), 3)) == 3
    assert len(seen) == 3 * 3 * 5 and set(seen) == {torch.float32}


@pytest.mark.parametrize("sinks", [0, 3])
def test_a_cache_grows(example, views, sinks):  # noqa: F811
    """Without a window a text has as many tokens as its caller likes: 4200 in pieces, as at once.

    In 32 bits: sums of up to 2000 terms by matrices and of 4200 by attention, twice in three layers, are off by less than
    2 (2000 + 3 * 2 * 4200) 2^-24 < 2^-8 of the largest logit."""
    tokens = text(4200)
    model = example.Decoder(views, torch.float32, None, sinks)
    with torch.no_grad():
        want = model.logits(tokens)
        cache, got, at = example.Cache(model), [], 0
        for n in (1, 1, 700, 1, 3390, 1, 1, 1, 1, 103):
            got.append(model.logits(tokens[at:at + n], cache))
            at += n
    assert at == 4200 and (torch.cat(got) - want).abs().max() <= 2.0 ** -8 * want.abs().max()


def test_an_answer_past_4096_tokens(example, views):  # noqa: F811
    model = example.Decoder(views)
    assert model.answer(text(4094), 6).shape == (6,)


def test_steps_wait_for_nothing(example, views):  # noqa: F811
    """A prompt's pieces and single tokens copy nothing from the host and read nothing back."""
    model = example.Decoder(views, window=20, sinks=2)
    tokens = text(64)
    with torch.no_grad():
        torch.cuda.set_sync_debug_mode("error")
        try:
            cache = example.Cache(model)
            for n in (30, 1, 1, 5):
                model.logits(tokens[:n], cache)
        finally:
            torch.cuda.set_sync_debug_mode("default")
