"""Serve and tune a loaded checkpoint whose matrices are kept in four bits.

A small decoder with the tensor names of the Llama checkpoints, random weights:
it is converted and loaded into HBM, its matrices are quantised there, and the
16-bit image is freed.  Then

* a prompt is answered, one token at a time after the prompt itself, over a cache
  that holds the last ``--window`` tokens and the first ``--sinks`` (``embedding``,
  ``rms_norm``, ``mx4_linear``, ``attention_cached``; with ``--mx4-prompt`` or
  ``--mx8-prompt`` the prompt's activations are in four or eight bits too);
* the embedding table is tuned to a text while the matrices stay as they are
  (``attention``; the backward passes are the operators').

    python examples/mx4_decoder.py [--layers 4] [--dim 1024] [--answer 32] [--steps 20] [--mx4-prompt | --mx8-prompt]
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


def rotate(x, first: int):
    """Rotary positions from ``first`` on: x is (tokens, heads, HEAD), the result in 32 bits."""
    angle = torch.arange(first, first + x.shape[0], device=x.device, dtype=torch.float32)[:, None, None] \
        * torch.pow(10000.0, -torch.arange(0, HEAD, 2, device=x.device, dtype=torch.float32) / HEAD)
    a, b = x[..., :HEAD // 2].float(), x[..., HEAD // 2:].float()
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


class Cache:
    """The keys and values of one sequence, layer by layer, in 32 bits, and how many tokens it has had."""

    def __init__(self, model: "Decoder"):
        self.past, self.room, self.grows = 0, model.window or 1, not model.window
        self.lengths = torch.zeros(1, dtype=torch.int64, device=model.table.device)
        self.layers = [self._empty(model) for _ in model.layers]

    def _empty(self, model: "Decoder"):
        return operators.KvCache.empty(1, model.kv_heads, HEAD, self.room, model.sinks, dtype=torch.float32, device=model.table.device)

    def reserve(self, model: "Decoder", n: int):
        """Room for n tokens more: a window's is all there ever is, and without one the layers grow."""
        if not self.grows or self.past + n <= self.room:
            return
        self.room = max(self.past + n, 2 * self.room)
        for i, old in enumerate(self.layers):
            new = self.layers[i] = self._empty(model)
            for to, held in ((new.k, old.k), (new.v, old.v)):
                to[:, :, :self.past] = held[:, :, :self.past]  # none has gone round: position p is in slot p

    def advance(self, n: int):
        self.past += n
        self.lengths += n


class Decoder:
    """The matrices in MX FP4, activations and the embedding table in ``dtype``."""

    def __init__(self, views, dtype=torch.bfloat16, window=None, sinks: int = 0):
        self.dtype, self.window, self.sinks = dtype, window, sinks
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

    def product(self, x, w, bits=None):
        if bits and not isinstance(x, operators.Mx8):
            x = (operators.mx4_quantize if bits == 4 else operators.mx8_quantize)(x)
        return operators.mx4_linear(x, w, out_dtype=self.dtype)

    def attention(self, qkv, cache, layer: int, offsets=None):
        """Causal attention of the new tokens over the cache's and themselves, in 32 bits."""
        kv = self.kv_heads * HEAD
        q, k, v = (y.unflatten(-1, (-1, HEAD)) for y in qkv.split([self.dim, kv, kv], -1))
        past = 0 if cache is None else cache.past
        q, k, v = rotate(q, past), rotate(k, past), v.float()
        if cache is None:
            out = operators.attention(q, k, v, window=self.window, sinks=self.sinks)
        else:
            out = operators.attention_cached(q, k, v, cache.layers[layer], cache.lengths, offsets=offsets)
        return out.flatten(1).to(self.dtype)

    def logits(self, tokens, cache=None, mx4: bool = False, table=None, bits=None):
        """(tokens, vocab); ``cache`` is a :class:`Cache`; ``bits`` (4 or 8, or ``mx4``) is what
        activations have in products."""
        bits = 4 if mx4 else bits
        n, offsets = len(tokens), None
        if cache is not None:
            cache.reserve(self, n)
            if n != 1:  # where the new tokens start and end, made on the GPU
                offsets = torch.arange(2, dtype=torch.int32, device=tokens.device) * n
        x = operators.embedding(self.table if table is None else table, tokens)
        new = None  # what the layer before has added

        def norm(gain):
            nonlocal x
            if new is None:
                return operators.rms_norm(x, gain, mx8=bits == 8)
            y, x = operators.rms_norm(new, gain, residual=x, mx8=bits == 8)
            return y

        for i, l in enumerate(self.layers):
            a = self.attention(self.product(norm(l["norm1"]), l["qkv"], bits), cache, i, offsets)
            new = self.product(a, l["out"], bits)
            gate, up = self.product(norm(l["norm2"]), l["gate_up"], bits).chunk(2, -1)
            new = self.product(torch.nn.functional.silu(gate) * up, l["down"], bits)
        if cache is not None:
            cache.advance(n)
        return self.product(norm(self.norm), self.head, bits)

    def answer(self, prompt, n: int, mx4_prompt: bool = False, bits=None):
        """The n most likely tokens after the prompt, one after the other."""
        cache, out = Cache(self), []
        with torch.no_grad():
            for _ in range(n):
                logits = self.logits(out[-1], cache) if out else self.logits(prompt, cache, mx4_prompt, bits=bits)
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
    ap.add_argument("--window", type=int, help="tokens that attention looks back, all of them if not given")
    ap.add_argument("--sinks", type=int, default=0, help="first tokens that stay visible")
    bits = ap.add_mutually_exclusive_group()
    bits.add_argument("--mx4-prompt", dest="bits", action="store_const", const=4)
    bits.add_argument("--mx8-prompt", dest="bits", action="store_const", const=8)
    a = ap.parse_args()

    spec = checkpoint(a.layers, a.dim, a.ffn, a.vocab, max(1, a.dim // HEAD // 4))
    with tempfile.TemporaryDirectory() as d:
        views = load(spec, os.path.join(d, "ckpt"))
    image = sum(v.numel() * v.element_size() for v in views.values())
    model = Decoder(views, window=a.window, sinks=a.sinks)
    held = sum(w.nbytes for l in model.layers for w in l.values() if isinstance(w, operators.Mx4)) + model.head.nbytes
    del views
    print(f"loaded {image / 1e6:.1f} MB; the matrices take {held / 1e6:.1f} MB in four bits")

    prompt = torch.randint(a.vocab, (a.prompt,), device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1))
    model.answer(prompt, 2, bits=a.bits)  # first calls load code
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    answer = model.answer(prompt, a.answer, bits=a.bits).tolist()
    print(f"{a.prompt} + {a.answer} tokens in {1e3 * (time.perf_counter() - t0):.1f} ms: {answer}")

    losses = model.tune(prompt, a.steps, rate=100.0)
    if losses:
        print("loss of the text while its embeddings are tuned: " + " ".join(f"{x:.3f}" for x in losses))


if __name__ == "__main__":
    main()
