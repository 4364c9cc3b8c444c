"""Serve and tune a loaded checkpoint whose matrices are kept in four bits.

A small decoder with the tensor names of the Llama checkpoints, random weights:
it is converted and loaded into HBM, its matrices are quantised there, and the
16-bit image is freed.  Then

* a prompt is answered, one token at a time after the prompt itself
  (``embedding``, ``mx4_linear``; with ``--mx4-prompt`` the prompt's
  activations are in four bits too);
* the embedding table is tuned to a text while the matrices stay as they are
  (the backward passes are ``mx4_linear_grad`` and ``embedding_grad``).

    python examples/mx4_decoder.py [--layers 4] [--dim 1024] [--answer 32] [--steps 20] [--mx4-prompt]
"""

from __future__ import annotations

import argparse
import os
import sys
import tempfile
import time

import torch

if __name__ == "__main__":  # from a checkout
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2401_14351_amd import binding, operators, synth

HEAD = 64  # elements of an attention head


def checkpoint(layers: int, dim: int, ffn: int, vocab: int, kv_heads: int, seed: int = 7) -> synth.CheckpointSpec:
    """The tensors of a decoder, bf16."""
    kv = kv_heads * HEAD
    t = [synth.TensorSpec("model.embed_tokens.weight", "bf16", (vocab, dim))]
    for layer in range(layers):
        p = f"model.layers.{layer}."
        for name, shape in (("self_attn.q_proj", (dim, dim)), ("self_attn.k_proj", (kv, dim)),
                            ("self_attn.v_proj", (kv, dim)), ("self_attn.o_proj", (dim, dim)),
                            ("mlp.gate_proj", (ffn, dim)), ("mlp.up_proj", (ffn, dim)), ("mlp.down_proj", (dim, ffn))):
            t.append(synth.TensorSpec(f"{p}{name}.weight", "bf16", shape))
        t.append(synth.TensorSpec(p + "input_layernorm.weight", "bf16", (dim,), init="ones"))
        t.append(synth.TensorSpec(p + "post_attention_layernorm.weight", "bf16", (dim,), init="ones"))
    t.append(synth.TensorSpec("model.norm.weight", "bf16", (dim,), init="ones"))
    t.append(synth.TensorSpec("lm_head.weight", "bf16", (vocab, dim)))
    return synth.CheckpointSpec("mx4-decoder", seed, alignment=256, chunk_size=1 << 20, tensors=t)


def load(spec: synth.CheckpointSpec, directory: str):
    """Convert the checkpoint into ``directory`` and load it: its views by name."""
    binding.convert([(t.name, t.dtype, t.shape, synth.tensor_bytes(spec, i)) for i, t in enumerate(spec.tensors)],
                    directory, alignment=spec.alignment, chunk_size=spec.chunk_size)
    return binding.load(directory, device=0)[1]


def stacked(*parts: torch.Tensor) -> operators.Mx4:
    """Matrices of equal columns as one, so that one product serves them all."""
    w = operators.Mx4.empty(sum(p.shape[0] for p in parts), parts[0].shape[1], parts[0].device)
    row = 0
    for p in parts:
        operators.mx4_quantize(p, out=w[row:row + p.shape[0]])
        row += p.shape[0]
    return w


def norm(x, gain, eps=1e-5):
    h = x.float()
    return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * gain).to(x.dtype)


def rotate(x, first: int):
    """Rotary positions from ``first`` on: x is (heads, tokens, HEAD) in 32 bits."""
    angle = torch.arange(first, first + x.shape[1], device=x.device, dtype=torch.float32)[:, None] \
        * torch.pow(10000.0, -torch.arange(0, HEAD, 2, device=x.device, dtype=torch.float32) / HEAD)
    a, b = x[..., :HEAD // 2], x[..., HEAD // 2:]
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


class Decoder:
    """The matrices in MX FP4, activations and the embedding table in ``dtype``."""

    def __init__(self, views, dtype=torch.bfloat16):
        self.dtype = dtype
        self.table = views["model.embed_tokens.weight"].to(dtype, copy=True)
        self.dim = self.table.shape[1]
        self.layers = []
        while f"model.layers.{len(self.layers)}.input_layernorm.weight" in views:
            p = f"model.layers.{len(self.layers)}."
            qkv = [views[f"{p}self_attn.{m}_proj.weight"] for m in "qkv"]
            self.kv_heads = qkv[1].shape[0] // HEAD
            self.layers.append({
                "qkv": stacked(*qkv), "out": stacked(views[p + "self_attn.o_proj.weight"]),
                "gate_up": stacked(views[p + "mlp.gate_proj.weight"], views[p + "mlp.up_proj.weight"]),
                "down": stacked(views[p + "mlp.down_proj.weight"]),
                "norm1": views[p + "input_layernorm.weight"].float(),
                "norm2": views[p + "post_attention_layernorm.weight"].float()})
        self.norm = views["model.norm.weight"].float()
        self.head = stacked(views["lm_head.weight"])

    def product(self, x, w, mx4: bool):
        if mx4:
            return operators.mx4_linear(operators.mx4_quantize(x), w, out_dtype=self.dtype)
        return operators.mx4_linear(x, w)

    def attention(self, qkv, cache, layer: int):
        """Causal attention of the new tokens over the cache's and themselves, in 32 bits."""
        t, kv = qkv.shape[0], self.kv_heads * HEAD
        q, k, v = (y.float().view(t, -1, HEAD).transpose(0, 1) for y in qkv.split([self.dim, kv, kv], -1))
        past = cache[layer][0].shape[1] if cache is not None and layer in cache else 0
        q, k = rotate(q, past), rotate(k, past)
        if past:
            k, v = torch.cat([cache[layer][0], k], 1), torch.cat([cache[layer][1], v], 1)
        if cache is not None:
            cache[layer] = (k, v)
        group = q.shape[0] // self.kv_heads
        k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
        score = torch.matmul(q, k.transpose(1, 2).contiguous()) * HEAD ** -0.5
        ahead = torch.ones(t, past + t, dtype=torch.bool, device=q.device).triu(past + 1)
        p = torch.softmax(score.masked_fill(ahead, float("-inf")), -1)
        return torch.matmul(p, v.contiguous()).transpose(0, 1).reshape(t, self.dim).to(self.dtype)

    def logits(self, tokens, cache=None, mx4: bool = False, table=None):
        """(tokens, vocab); ``cache`` is a dict that keeps the keys and values of a sequence."""
        x = operators.embedding(self.table if table is None else table, tokens)
        for i, l in enumerate(self.layers):
            a = self.attention(self.product(norm(x, l["norm1"]), l["qkv"], mx4), cache, i)
            x = x + self.product(a, l["out"], mx4)
            gate, up = self.product(norm(x, l["norm2"]), l["gate_up"], mx4).chunk(2, -1)
            x = x + self.product(torch.nn.functional.silu(gate) * up, l["down"], mx4)
        return self.product(norm(x, self.norm), self.head, mx4)

    def answer(self, prompt, n: int, mx4_prompt: bool = False):
        """The n most likely tokens after the prompt, one after the other."""
        cache, out = {}, []
        with torch.no_grad():
            for _ in range(n):
                logits = self.logits(out[-1], cache) if out else self.logits(prompt, cache, mx4_prompt)
                out.append(logits[-1].argmax().view(1))
        return torch.cat(out) if out else prompt[:0]

    def tune(self, text, steps: int, rate: float):
        """Fit the table to a text, the matrices fixed; the loss before each step."""
        master = self.table.float()  # small steps would round away in 16 bits
        losses = []
        for _ in range(steps):
            table = master.to(self.dtype).requires_grad_()
            loss = torch.nn.functional.cross_entropy(self.logits(text[:-1], table=table).float(), text[1:].long())
            loss.backward()
            losses.append(loss.detach())
            master -= rate * table.grad.float()
        self.table = master.to(self.dtype)
        return torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--dim", type=int, default=1024)
    ap.add_argument("--ffn", type=int, default=2816)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--answer", type=int, default=32)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--mx4-prompt", action="store_true")
    a = ap.parse_args()

    spec = checkpoint(a.layers, a.dim, a.ffn, a.vocab, max(1, a.dim // HEAD // 4))
    with tempfile.TemporaryDirectory() as d:
        views = load(spec, os.path.join(d, "ckpt"))
    image = sum(v.numel() * v.element_size() for v in views.values())
    model = Decoder(views)
    held = sum(w.nbytes for l in model.layers for w in l.values() if isinstance(w, operators.Mx4)) + model.head.nbytes
    del views
    print(f"loaded {image / 1e6:.1f} MB; the matrices take {held / 1e6:.1f} MB in four bits")

    prompt = torch.randint(a.vocab, (a.prompt,), device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1))
    model.answer(prompt, 2, a.mx4_prompt)  # first calls load code
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    answer = model.answer(prompt, a.answer, a.mx4_prompt).tolist()
    print(f"{a.prompt} + {a.answer} tokens in {1e3 * (time.perf_counter() - t0):.1f} ms: {answer}")

    losses = model.tune(prompt, a.steps, rate=100.0)
    if losses:
        print("loss of the text while its embeddings are tuned: " + " ".join(f"{x:.3f}" for x in losses))


if __name__ == "__main__":
    main()
