"""The decoder example: convert, load, quantise in HBM, answer and tune, against
the same decoder in 64 bits on the CPU with the values the four bits stand for."""

import importlib.util
import math
import os

import numpy as np
import pytest

from oracle import operators_oracle as oo
from paper_2401_14351_amd import synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LAYERS, DIM, FFN, VOCAB, KV_HEADS = 2, 192, 200, 517, 1

# 32-bit rounding, in units of the largest value: a step that sums n terms in 32
# bits is off by at most n * 2^-24 of the sum of magnitudes.  The depths on the
# way to a logit add up to under 2 * (3 * 192 + 200 + 2 * 64) + 192 = 2000, the
# norms at most double what reaches them: 2 * 2000 * 2^-24 = 2^-12.  A gradient
# goes the way back too, and through the softmax of the loss: four times that.
LOGIT_TOL, GRAD_TOL = 2.0 ** -12, 2.0 ** -10


@pytest.fixture(scope="module")
def example():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    found = importlib.util.spec_from_file_location("mx4_decoder", os.path.join(ROOT, "examples", "mx4_decoder.py"))
    module = importlib.util.module_from_spec(found)
    found.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def spec(example):
    return example.checkpoint(LAYERS, DIM, FFN, VOCAB, KV_HEADS)


@pytest.fixture(scope="module")
def views(example, spec, tmp_path_factory):
    return example.load(spec, str(tmp_path_factory.mktemp("decoder") / "ckpt"))


@pytest.fixture(scope="module")
def exact(spec):
    """The checkpoint's values in 64 bits, its matrices as their four bits have them."""
    import torch

    out = {}
    for i, t in enumerate(spec.tensors):
        raw = synth.tensor_bytes(spec, i).view(np.uint16).astype(np.uint32) << 16
        v = raw.view(np.float32).reshape(t.shape).astype(np.float64)
        if len(t.shape) == 2 and "embed" not in t.name:
            v = oo.dequantize(*oo.quantize(v), v.shape[1])
        out[t.name] = torch.from_numpy(v)
    return out


def logits64(torch, w, table, tokens):
    def norm(x, g):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * g

    def heads(y):
        return y.reshape(len(tokens), -1, 64).transpose(0, 1)

    freq = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    angle = torch.arange(len(tokens), dtype=torch.float64)[:, None] * freq
    turn = torch.polar(torch.ones_like(angle), angle)

    def rotate(y):
        z = torch.complex(y[..., :32].contiguous(), y[..., 32:].contiguous()) * turn
        return torch.cat([z.real, z.imag], -1)

    x = table[tokens]
    for i in range(LAYERS):
        p = f"model.layers.{i}."
        h = norm(x, w[p + "input_layernorm.weight"])
        q, k, v = (heads(h @ w[f"{p}self_attn.{m}_proj.weight"].T) for m in "qkv")
        s = rotate(q) @ rotate(k).transpose(1, 2) / 8
        s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool).triu(1), -math.inf)
        a = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(len(tokens), DIM)
        x = x + a @ w[p + "self_attn.o_proj.weight"].T
        h = norm(x, w[p + "post_attention_layernorm.weight"])
        g = h @ w[p + "mlp.gate_proj.weight"].T
        x = x + (g * torch.sigmoid(g) * (h @ w[p + "mlp.up_proj.weight"].T)) @ w[p + "mlp.down_proj.weight"].T
    return norm(x, w["model.norm.weight"]) @ w["lm_head.weight"].T


def text(torch, n, seed):
    return torch.randint(VOCAB, (n,), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("n", [1, 17, 70])
def test_logits(example, views, exact, n):
    import torch

    tokens = text(torch, n, n)
    model = example.Decoder(views, torch.float32)
    got = model.logits(tokens.cuda()).double().cpu()
    want = logits64(torch, exact, exact["model.embed_tokens.weight"], tokens)
    assert (got - want).abs().max() <= LOGIT_TOL * want.abs().max()


def test_answer_token_by_token(example, views, exact):
    """Every token of the answer is the most likely one after those before it."""
    import torch

    prompt = text(torch, 23, 5)
    model = example.Decoder(views, torch.float32)
    answer = model.answer(prompt.cuda(), 6).cpu()
    whole = logits64(torch, exact, exact["model.embed_tokens.weight"], torch.cat([prompt, answer]))
    for i in range(6):
        row = whole[22 + i]
        assert row[answer[i]] >= row.max() - 2 * LOGIT_TOL * row.abs().max()


def test_table_gradient(example, views, exact):
    import torch

    tokens = text(torch, 40, 9)
    tokens[20:25] = tokens[3]  # a token that comes up often
    model = example.Decoder(views, torch.float32)
    table = model.table.clone().requires_grad_()
    loss = torch.nn.functional.cross_entropy(model.logits(tokens[:-1].cuda(), table=table), tokens[1:].cuda())
    loss.backward()
    table64 = exact["model.embed_tokens.weight"].clone().requires_grad_()
    loss64 = torch.nn.functional.cross_entropy(logits64(torch, exact, table64, tokens[:-1]), tokens[1:])
    loss64.backward()
    got, want = table.grad.double().cpu(), table64.grad
    assert abs(loss.item() - loss64.item()) <= LOGIT_TOL * abs(loss64.item())
    assert (got - want).abs().max() <= GRAD_TOL * want.abs().max()
    unused = torch.ones(VOCAB, dtype=torch.bool)
    unused[tokens[:-1]] = False
    assert not got[unused].any()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_tuning_lowers_the_loss(example, views, dtype):
    import torch

    model = example.Decoder(views, getattr(torch, dtype))
    losses = model.tune(text(torch, 64, 3).cuda(), 8, rate=5.0)
    assert all(math.isfinite(x) for x in losses) and losses[-1] < losses[0]


def test_prompt_in_four_bits(example, views, exact):
    """An element is rounded by at most a quarter of itself down to a twelfth of
    its block's largest, a tenth or less on average; seven products in a row of
    the residual stream and the head's keep the logits within six tenths."""
    import torch

    tokens = text(torch, 50, 11)
    model = example.Decoder(views)
    got = model.logits(tokens.cuda(), mx4=True)
    assert got.dtype == torch.bfloat16 and torch.equal(got, model.logits(tokens.cuda(), mx4=True))
    want = logits64(torch, exact, exact["model.embed_tokens.weight"], tokens)
    assert (got.double().cpu() - want).norm() <= 0.6 * want.norm()
