"""Operators of a decoder layer around its four-bit matrices, as measurable cases.

What a layer does between the products with loaded weights, for tuning a model
and for serving it:

* ``attention``    causal attention over packed sequences, with a sliding window
                   and a few first tokens that stay visible (sinks): query i sees
                   key j where j <= i and (i - j < window or j < sinks).  Key/value
                   heads are shared by groups of query heads.
* ``attention_train``  the same with its backward pass.
* ``step``         one new token a sequence, over a cache that holds the sinks and
                   the window: position p is in slot p, or, from the sinks on, in
                   slot sinks + (p - sinks) % window.  The token is written too.
* ``chunk``        pieces of prompts over the same cache: they see what it holds
                   and themselves, and are written after.
* ``norm``         h = x + residual, rounded to their type, and h over its root
                   mean square, times a gain.
* ``norm_train``   the same with its backward pass.
* ``norm_linear8`` h, and the product of its norm in MX FP8 (blocks of 32 along a
                   row, one power-of-two scale a block, E4M3 elements) with a
                   weight in MX FP4.

Heads and widths are those of the synthetic checkpoints: OPT-125M (12 heads of 64),
Llama-2 7B / 13B / 70B shaped ones (32 and 40 heads of 128; 64 that share 8 key/value
heads; widths 4096 / 5120 / 8192, feed forward 11008 / 13824 / 28672, 1024 key/value
columns in the 70B).
"""

import math

import torch

own = False

BLOCK = 32          # values that share a scale
EPS = 1e-5
_DEVICE = "cuda"
_TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # one short OPT-125M prompt, every token visible: bound by latency
        {"name": "attention short f16", "do": "attention", "tokens": 77, "sequences": 1, "heads": 12, "kv_heads": 12,
         "dim": 64, "window": 0, "sinks": 0, "type": "f16"},
        # prompts of the 7B packed one behind the other, of lengths that are no round numbers
        {"name": "attention packed bf16", "do": "attention", "tokens": 8191, "sequences": 5, "heads": 32, "kv_heads": 32,
         "dim": 128, "window": 1024, "sinks": 4, "type": "bf16"},
        # one long prompt of the 70B
        {"name": "attention long bf16", "do": "attention", "tokens": 16384, "sequences": 1, "heads": 64, "kv_heads": 8,
         "dim": 128, "window": 4096, "sinks": 4, "type": "bf16"},
        # a tuning step of the 7B over four texts
        {"name": "attention_train bf16", "do": "attention_train", "tokens": 8192, "sequences": 4, "heads": 32,
         "kv_heads": 32, "dim": 128, "window": 1024, "sinks": 4, "type": "bf16"},
        # a ragged last micro-batch in half precision, shared heads of an odd group
        {"name": "attention_train ragged f16", "do": "attention_train", "tokens": 1333, "sequences": 3, "heads": 15,
         "kv_heads": 5, "dim": 80, "window": 300, "sinks": 2, "type": "f16"},
        # decoding one sequence of the 70B a hundred thousand tokens long
        {"name": "step long bf16", "do": "step", "sequences": 1, "heads": 64, "kv_heads": 8, "dim": 128,
         "window": 131072, "sinks": 4, "past": 100003, "type": "bf16"},
        # decoding a batch of the 7B, its sequences of all lengths
        {"name": "step batch f16", "do": "step", "sequences": 32, "heads": 32, "kv_heads": 32, "dim": 128,
         "window": 1024, "sinks": 4, "past": 5000, "type": "f16"},
        # pieces of prompts of the 70B beside sequences that have one token or none
        {"name": "chunk bf16", "do": "chunk", "tokens": 1200, "sequences": 8, "heads": 64, "kv_heads": 8, "dim": 128,
         "window": 2048, "sinks": 4, "past": 800, "type": "bf16"},
        # decoding one token: the smallest norm
        {"name": "norm token bf16", "do": "norm", "rows": 1, "cols": 4096, "type": "bf16"},
        # a tuning step of the 13B
        {"name": "norm_train bf16", "do": "norm_train", "rows": 8191, "cols": 5120, "type": "bf16"},
        # decoding a batch: the 70B's key projection behind its norm
        {"name": "norm_linear8 tokens bf16", "do": "norm_linear8", "rows": 16, "cols": 8192, "out": 1024, "type": "bf16"},
        # 4096 positions through the 70B's up projection
        {"name": "norm_linear8 prompt bf16", "do": "norm_linear8", "rows": 4096, "cols": 8192, "out": 28672,
         "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    do = rng.choice(["attention", "attention_train", "step", "chunk", "norm", "norm_train", "norm_linear8"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])

    def width(lo, hi):  # a width of the checkpoints, or any other
        known = [w for w in (768, 1024, 4096, 5120, 8192, 11008, 13824, 28672) if lo <= w <= hi]
        return rng.choice(known) if rng.random() < 0.4 else _log_int(rng, lo, hi)

    if do in ("norm", "norm_train"):
        return {"do": do, "rows": _log_int(rng, 1, 16384), "cols": width(65, 13824 if do == "norm" else 8192), "type": kind}
    if do == "norm_linear8":
        return {"do": do, "rows": _log_int(rng, 1, 4096), "cols": width(65, 13824), "out": width(65, 13824), "type": kind}
    heads, kv_heads, dim = rng.choice([(12, 12, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), None]) or (0, 0, 0)
    if not heads:
        kv_heads = rng.randint(1, 8)
        heads, dim = kv_heads * rng.randint(1, 8), rng.choice([64, 128, 8 * rng.randint(2, 16), rng.randint(16, 128)])
    case = {"do": do, "heads": heads, "kv_heads": kv_heads, "dim": dim, "sinks": rng.choice([0, 1, 4, rng.randint(0, 200)]),
            "type": kind}
    if do in ("attention", "attention_train"):
        case["tokens"] = _log_int(rng, 1, 16384)
        case["sequences"] = rng.randint(1, max(1, min(16, case["tokens"] // 4)))
        case["window"] = rng.choice([0, _log_int(rng, 1, 8192)])
        while work(case)["flops"] > (1.0e12 if kind != "f32" else 1.5e11):
            case["tokens"] = case["tokens"] // 2 + 1
        return case
    case["sequences"] = _log_int(rng, 1, 64)
    limit = 4e8  # elements of the cache
    case["window"] = _log_int(rng, 1, max(1, min(131072, int(limit / (case["sequences"] * kv_heads * dim)) - case["sinks"])))
    if do == "step":  # a window still filling, or gone round many times
        case["past"] = _log_int(rng, 1, 3 * case["window"] + 10) - 1
        return case
    # a chunk that still leaves room, so that the same call can be made again
    room = case["sinks"] + case["window"]
    case["tokens"] = _log_int(rng, 1, min(8192, room * case["sequences"]))
    while max(_tokens_of(case)) > room:
        case["tokens"] //= 2
    case["past"] = rng.randint(0, room - max(_tokens_of(case)))
    return case


# ---------------------------------------------------------------------------
# what a case's sequences hold
# ---------------------------------------------------------------------------

def _spread(i):
    return i * 0.6180339887498949 % 1.0


def _tokens_of(case):
    """New tokens of each sequence: uneven pieces, and of a chunk's sequences some
    have one token or none."""
    n, total = case["sequences"], case["tokens"]
    weight = [0.4 + _spread(i + 1) for i in range(n)]
    if case["do"] == "chunk":
        weight = [0.0 if n > 2 and i % 4 == 2 else w for i, w in enumerate(weight)]
    single = [i for i in range(n) if case["do"] == "chunk" and n > 2 and i % 4 == 1]
    rest = max(0, total - len(single))
    whole = sum(w for i, w in enumerate(weight) if i not in single)
    out = [0 if i in single else int(rest * w / whole) for i, w in enumerate(weight)]
    for i in single[:total]:
        out[i] = 1
    left = [i for i, w in enumerate(weight) if w and i not in single]
    for i in range(total - sum(out)):
        out[left[i % len(left)]] += 1
    return out


def _past_of(case):
    """Tokens that each sequence has had before: the first one's is the most."""
    return [int(case["past"] * (1 - 0.9 * _spread(i))) for i in range(case["sequences"])]


def _seen(at, window, sinks):
    """How many keys the query at a position sees."""
    return at + 1 if not window or at < window else window + min(sinks, at + 1 - window)


def _pairs(first, n, window, sinks):
    """Visible keys of the queries at first .. first + n - 1, together."""
    if not window:
        return n * first + n * (n + 1) // 2
    total = 0
    grow = max(0, min(first + n, window) - first)     # at < window
    total += grow * first + grow * (grow + 1) // 2
    first, n = first + grow, n - grow
    part = max(0, min(first + n, window + sinks) - first)  # not all sinks are behind the window yet
    total += part * (first + 1) + part * (part - 1) // 2
    return total + (n - part) * (window + sinks)


# ---------------------------------------------------------------------------
# MX FP4 and MX FP8 in elementary operations
# ---------------------------------------------------------------------------

def _blocks(x):
    """x, its rows padded with zeros to whole blocks."""
    rows, cols = x.shape
    out = torch.zeros(rows, -(-cols // BLOCK) * BLOCK, dtype=x.dtype, device=x.device)
    out[:, :cols] = x
    return out.view(rows, -1, BLOCK)


def _times_power(x, e):
    """x times 2^e in two steps, neither of which leaves the type's range before the result does."""
    return torch.ldexp(torch.ldexp(x, e // 2), e - e // 2)


def _fp8_values(x):
    """The values that x in 32 bits becomes in MX FP8.  A block's exponent is the
    smallest, from -127 on, whose 448-fold holds its largest magnitude."""
    b = _blocks(x)
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (m > 0.875), torch.full_like(e, -127)).clamp(min=-127)
    y = _times_power(b, -e)
    step = torch.frexp(y)[1].clamp(min=-5) - 4  # of three bits behind the leading one, down to 2^-9
    v = _times_power(torch.ldexp(torch.round(torch.ldexp(y, -step)), step), e)
    return v.reshape(x.shape[0], -1)[:, :x.shape[1]]


def _fp4_pack(x):
    """Codes and scales of x as they are stored: two codes a byte, the even column in
    the low half, 16 bytes a block; a row's scale bytes padded to a multiple of 16."""
    b = _blocks(x)
    e = torch.frexp(b.abs().amax(-1))[1] - 3
    y = torch.ldexp(b.abs(), -e.unsqueeze(-1))
    code = torch.where(y < 2, torch.round(y * 2), torch.where(y < 4, torch.round(y) + 2, torch.round(y / 2) + 4))
    code = code.clamp(max=7).to(torch.uint8) | (torch.signbit(b).to(torch.uint8) << 3)
    rows, nb = e.shape
    scales = torch.zeros(rows, -(-nb // 16) * 16, dtype=torch.uint8, device=x.device)
    scales[:, :nb] = (e + 127).to(torch.uint8)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(rows, nb * 16), scales


def _fp4_values(codes, scales, cols, dtype):
    rows, nb = codes.shape[0], codes.shape[1] // 16
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype, device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], -1).view(rows, nb, BLOCK)
    v = level[code.to(torch.int32)] * torch.exp2(scales[:, :nb].to(dtype) - 127).unsqueeze(-1)
    return v.reshape(rows, -1)[:, :cols]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(shape, std, g):
    return torch.randn(shape, generator=g, device=_DEVICE) * std


def _stream(rows, cols, std, g):
    """Hidden states: most channels of one size, a few much larger."""
    gain = std * torch.exp(0.3 * torch.randn(cols, generator=g, device=_DEVICE))
    gain[torch.rand(cols, generator=g, device=_DEVICE) < 0.005] *= 12.0
    return _normal((rows, cols), 1.0, g) * gain


def _weight(rows, cols, g):
    parts = [_fp4_pack(_normal((min(4096, rows - r), cols), 0.02, g)) for r in range(0, rows, 4096)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _lengths(values, bits=torch.int32):
    return torch.tensor(values, dtype=bits, device=_DEVICE)


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed)
    do, kind = case["do"], _TYPE[case["type"]]
    state = {"case": case}
    if do.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        state["x"] = _stream(rows, cols, 0.2, g).to(kind)
        state["residual"] = _stream(rows, cols, 1.0, g).to(kind)
        state["gain"] = 1.0 + _normal((cols,), 0.1, g)
        if do == "norm_train":
            state["dy"] = _normal((rows, cols), 0.01, g).to(kind)
            state["dh"] = _normal((rows, cols), 0.01, g).to(kind)
            if own:
                for name in ("x", "residual", "gain"):
                    state[name].requires_grad_()
        if do == "norm_linear8":
            state["codes"], state["scales"] = _weight(case["out"], cols, g)
            if own:
                from paper_2401_14351_amd import operators

                state["mx4"] = operators.Mx4(state["codes"], state["scales"], cols)
        return state

    heads, kv_heads, dim, n = case["heads"], case["kv_heads"], case["dim"], case["sequences"]
    tokens = n if do == "step" else case["tokens"]
    # a row of the stacked projections holds a token's queries, keys and values
    rows = _normal((tokens, heads + 2 * kv_heads, dim), 1.0, g)
    rows[:, :heads] *= torch.exp(0.4 * torch.randn(heads, 1, generator=g, device=_DEVICE))  # some heads are sharper
    q, k, v = rows.to(kind).split([heads, kv_heads, kv_heads], 1)
    if do == "attention_train":  # rotated, so written out each on its own
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        state["dout"] = _normal((tokens, heads, dim), 0.02, g).to(kind)
        if own:
            for t in (q, k, v):
                t.requires_grad_()
    state.update(q=q, k=k, v=v)
    if do != "step" and (n > 1 or do == "chunk"):
        state["offsets"] = _lengths(_offsets(_tokens_of(case)))
    if do in ("step", "chunk"):
        slots = case["sinks"] + case["window"]
        for name in ("cache_k", "cache_v"):
            t = torch.empty(n, kv_heads, slots, dim, dtype=kind, device=_DEVICE)
            for i in range(n):
                t[i] = _normal((kv_heads, slots, dim), 1.0, g).to(kind)
            state[name] = t
        state["lengths"] = _lengths(_past_of(case))
        if own:
            from paper_2401_14351_amd import operators

            state["cache"] = operators.KvCache(state["cache_k"], state["cache_v"], case["window"], case["sinks"])
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2401_14351_amd import operators as op

    case = state["case"]
    do = case["do"]
    if do == "norm":
        return op.rms_norm(state["x"], state["gain"], residual=state["residual"], eps=EPS)
    if do == "norm_train":
        y, h = op.rms_norm(state["x"], state["gain"], residual=state["residual"], eps=EPS)
        grads = torch.autograd.grad((y, h), (state["x"], state["residual"], state["gain"]), (state["dy"], state["dh"]))
        return (y.detach(), h.detach(), *grads)
    if do == "norm_linear8":
        y, h = op.rms_norm(state["x"], state["gain"], residual=state["residual"], eps=EPS, mx8=True)
        return op.mx4_linear(y, state["mx4"], out_dtype=_TYPE[case["type"]]), h
    q, k, v = state["q"], state["k"], state["v"]
    if do in ("step", "chunk"):
        out = op.attention_cached(q, k, v, state["cache"], state["lengths"], offsets=state.get("offsets"))
        return out, state["cache"].k, state["cache"].v
    out = op.attention(q, k, v, window=case["window"] or None, sinks=case["sinks"], offsets=state.get("offsets"))
    if do == "attention":
        return out
    return (out.detach(), *torch.autograd.grad(out, (q, k, v), state["dout"]))


def _softmax(score, hidden):
    score = score.masked_fill(hidden, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _slots(first, n, case):
    """The slots of positions first .. first + n - 1."""
    p = torch.arange(first, first + n, device=_DEVICE)
    return torch.where(p < case["sinks"], p, case["sinks"] + (p - case["sinks"]) % case["window"])


def _pieces(first, n, window, sinks):
    """Runs of up to 1024 queries of a sequence from position `first` on: the run, the
    positions that some of it sees (sinks, then window), and what each must not see."""
    for r in range(0, n, 1024):
        rows = min(1024, n - r)
        at = torch.arange(first + r, first + r + rows, device=_DEVICE).unsqueeze(1)
        low = max(0, first + r - window + 1) if window else 0
        key = torch.cat([torch.arange(min(sinks, low), device=_DEVICE), torch.arange(low, first + r + rows, device=_DEVICE)])
        hidden = key > at
        if window:
            hidden |= (at - key >= window) & (key >= sinks)
        yield slice(r, r + rows), key, hidden


def _plain_attention(q, k, v, first, window, sinks, dout=None):
    """One sequence, in 32 bits: its new tokens' queries (from position `first` on) over
    all of its keys, heads first; the gradients too where dout is given."""
    kv_heads, group, n, dim = q.shape
    scale = dim ** -0.5
    out = torch.empty_like(q)
    if dout is not None:
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for h in range(kv_heads):
        for rows, key, hidden in _pieces(first, n, window, sinks):
            kk, vv = k[h, key], v[h, key]
            p = _softmax((q[h, :, rows] @ kk.t()) * scale, hidden)
            o = p @ vv
            out[h, :, rows] = o
            if dout is not None:
                do = dout[h, :, rows]
                ds = p * (do @ vv.t() - (do * o).sum(-1, keepdim=True)) * scale
                dq[h, :, rows] = ds @ kk
                dk[h].index_add_(0, key, (ds.transpose(1, 2).contiguous() @ q[h, :, rows].contiguous()).sum(0))
                dv[h].index_add_(0, key, (p.transpose(1, 2).contiguous() @ do.contiguous()).sum(0))
    return out if dout is None else (out, dq, dk, dv)


def _heads_first(t, groups):
    """(tokens, heads, dim) as (groups, heads of a group, tokens, dim) in 32 bits."""
    return t.detach().float().view(t.shape[0], groups, t.shape[1] // groups, t.shape[2]).permute(1, 2, 0, 3).contiguous()


def _tokens_first(t):
    return t.permute(2, 0, 1, 3).flatten(1, 2)


def _plain_packed(state):
    case, groups, kind = state["case"], state["case"]["kv_heads"], _TYPE[state["case"]["type"]]
    outs = []
    at = _offsets(_tokens_of(case))
    for a, b in zip(at, at[1:]):
        q, k, v = (_heads_first(state[t][a:b], groups) for t in "qkv")
        dout = _heads_first(state["dout"][a:b], groups) if case["do"] == "attention_train" else None
        got = _plain_attention(q, k[:, 0], v[:, 0], 0, case["window"], case["sinks"], dout)
        if dout is None:
            outs.append((_tokens_first(got),))
        else:
            outs.append((*(_tokens_first(t) for t in got[:2]), *(t.transpose(0, 1) for t in got[2:])))
    return tuple(torch.cat(parts).to(kind) for parts in zip(*outs))


def _plain_chunk(state):
    case, groups, kind = state["case"], state["case"]["kv_heads"], _TYPE[state["case"]["type"]]
    outs, at = [], _offsets(_tokens_of(case))
    for i, (a, b, past) in enumerate(zip(at, at[1:], _past_of(case))):
        q, k, v = (_heads_first(state[t][a:b], groups) for t in "qkv")
        held = _slots(0, past, case)
        keys, values = (torch.cat([state[c][i, :, held].float(), new[:, 0]], 1) for c, new in (("cache_k", k), ("cache_v", v)))
        outs.append(_tokens_first(_plain_attention(q, keys, values, past, case["window"], case["sinks"])))
        held = _slots(past, b - a, case)
        state["cache_k"][i, :, held] = state["k"][a:b].transpose(0, 1)
        state["cache_v"][i, :, held] = state["v"][a:b].transpose(0, 1)
    return torch.cat(outs).to(kind), state["cache_k"], state["cache_v"]


def _plain_step(state):
    case, groups = state["case"], state["case"]["kv_heads"]
    n, heads, dim = state["q"].shape
    sinks, window = case["sinks"], case["window"]
    t = state["lengths"].long()
    row = torch.arange(n, device=_DEVICE)
    at = torch.where(t < sinks, t, sinks + (t - sinks) % window)
    state["cache_k"][row, :, at] = state["k"]
    state["cache_v"][row, :, at] = state["v"]
    slot = torch.arange(sinks + window, device=_DEVICE)
    # the last position a slot of the window can hold, the token's own at most
    t = t.unsqueeze(1)
    held = torch.where(slot < sinks, slot <= t, t - (t - slot) % window >= sinks)
    out = torch.empty(n, groups, heads // groups, dim, device=_DEVICE)
    q = state["q"].float().view(out.shape)
    for i in range(n):
        score = (q[i] @ state["cache_k"][i].float().transpose(1, 2).contiguous()) * dim ** -0.5
        out[i] = _softmax(score, ~held[i]) @ state["cache_v"][i].float()
    return out.view(n, heads, dim).to(_TYPE[case["type"]]), state["cache_k"], state["cache_v"]


def _run_plain(state):
    case = state["case"]
    do = case["do"]
    kind = _TYPE[case["type"]]
    if do == "step":
        return _plain_step(state)
    if do == "chunk":
        return _plain_chunk(state)
    if do.startswith("attention"):
        out = _plain_packed(state)
        return out if do == "attention_train" else out[0]
    gain = state["gain"]
    h = (state["x"].float() + state["residual"].float()).to(kind)
    wide = h.float()
    r = torch.rsqrt((wide * wide).mean(-1, keepdim=True) + EPS)
    unit = wide * r
    y = unit * gain
    if do == "norm":
        return y.to(kind), h
    if do == "norm_linear8":
        return (_fp8_values(y) @ _fp4_values(state["codes"], state["scales"], case["cols"], torch.float32).t()).to(kind), h
    dy = state["dy"].float()
    s = dy * gain
    dx = (state["dh"].float() + r * (s - unit * (s * unit).mean(-1, keepdim=True))).to(kind)
    return y.to(kind), h, dx, dx, (dy * unit).sum(0)


# ---------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    do = case["do"]
    size = _SIZE[case["type"]]
    if do.startswith("norm"):
        n = case["rows"] * case["cols"]
        if do == "norm":
            return {"bytes": 4 * n * size + 4 * case["cols"], "flops": 5 * n}
        if do == "norm_train":
            return {"bytes": 7 * n * size + 8 * case["cols"], "flops": 14 * n}
        nb = -(-case["cols"] // BLOCK)
        return {"bytes": (3 * n + case["rows"] * case["out"]) * size + 4 * case["cols"] + case["out"] * nb * (BLOCK // 2 + 1),
                "flops": 2 * n * case["out"]}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    window, sinks = case["window"], case["sinks"]
    if do.startswith("attention"):
        pairs = sum(_pairs(0, n, window, sinks) for n in _tokens_of(case))
        each = case["tokens"] * (heads + kv_heads) * dim * size
        if do == "attention":
            return {"bytes": 2 * each, "flops": 4 * dim * heads * pairs}
        return {"bytes": 4 * each, "flops": 14 * dim * heads * pairs}
    past = _past_of(case)
    new = [1] * case["sequences"] if do == "step" else _tokens_of(case)
    pairs = sum(_pairs(p, n, window, sinks) for p, n in zip(past, new))
    # the past that some new token sees, once; new tokens in and into the cache
    held = sum(_seen(p, window, sinks) - 1 for p, n in zip(past, new) if n)
    row = 2 * kv_heads * dim * size
    return {"bytes": held * row + sum(new) * (2 * heads * dim * size + 2 * row), "flops": 4 * dim * heads * pairs}


def _nearest_fp8(x):
    """MX FP8 of x in 64 bits from the table of E4M3's values: what each element becomes."""
    code = torch.arange(127, device=x.device)
    exp, frac = code >> 3, (code & 7).double() / 8
    level = torch.where(exp == 0, frac * 2.0 ** -6, (1 + frac) * torch.exp2(exp.double() - 7))
    middle = (level[1:] + level[:-1]) / 2
    rows, cols = x.shape
    out = torch.empty_like(x)
    for r in range(0, rows, 1024):
        b = torch.nn.functional.pad(x[r:r + 1024], (0, -cols % BLOCK)).view(min(1024, rows - r), -1, BLOCK)
        top = b.abs().amax(-1, keepdim=True)
        power = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 9
        for _ in range(2):  # the smallest power whose 448-fold is not below the largest
            power = torch.where(torch.exp2(power) * 448 < top, power + 1, power)
        unit = torch.exp2(power.clamp(min=-127))
        y = (b.abs() / unit).contiguous()
        i = torch.searchsorted(middle, y)                  # how many middles lie below
        tie = (middle[i.clamp(max=125)] == y) & (i < 126)  # of two equally near, the even code
        i = i + (tie & (i % 2 == 1)).long()
        out[r:r + 1024] = (torch.copysign(level[i], b) * unit).view(b.shape[0], -1)[:, :cols]
    return out


def _exact_attention(q, k, v, at, key, case, dout=None):
    """Queries at positions `at` over keys at positions `key`, by their definition: one
    key/value head, every key and a mask."""
    seen = key.unsqueeze(0) <= at.unsqueeze(1)
    if case["window"]:
        seen &= (key.unsqueeze(0) + case["window"] > at.unsqueeze(1)) | (key.unsqueeze(0) < case["sinks"])
    scale = 1 / math.sqrt(q.shape[-1])
    outs, dqs, dk, dv = [], [], torch.zeros_like(k), torch.zeros_like(v)
    for i in range(q.shape[1]):  # the heads that share these keys
        x = (scale * q[:, i]) @ k.T.contiguous()
        weight = torch.where(seen, torch.exp(x - torch.where(seen, x, -math.inf).max(1, keepdim=True).values), 0.0)
        weight /= weight.sum(1, keepdim=True)
        outs.append(weight @ v)
        if dout is not None:
            inner = dout[:, i] @ v.T.contiguous()
            inner = weight * (inner - (weight * inner).sum(1, keepdim=True)) * scale
            dqs.append(inner @ k)
            dk += inner.T.contiguous() @ q[:, i]
            dv += weight.T.contiguous() @ dout[:, i]
    out = torch.stack(outs, 1)
    return (out,) if dout is None else (out, torch.stack(dqs, 1), dk, dv)


def _exact_heads(state, tokens, keys, values, at, key, dout=None):
    """_exact_attention of every key/value head, runs of queries at a time."""
    case = state["case"]
    group = case["heads"] // case["kv_heads"]
    got = []
    for h in range(case["kv_heads"]):
        mine = slice(h * group, (h + 1) * group)
        q = state["q"].detach()[tokens, mine].double()
        k, v = keys[:, h].double(), values[:, h].double()
        parts = []
        for r in range(0, len(at), 4096):
            rows = slice(r, r + 4096)
            last = int(at[rows][-1]) if len(key) else 0
            low = key <= last
            if case["window"]:
                low &= (key + case["window"] > int(at[rows][0])) | (key < case["sinks"])
            low = torch.nonzero(low).flatten()
            part = _exact_attention(q[rows].contiguous(), k[low], v[low], at[rows], key[low], case,
                                    None if dout is None else dout[rows, mine].double())
            parts.append((low, part))
        whole = [torch.cat([p[0] for _, p in parts])]
        if dout is not None:
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            for low, p in parts:
                dk[low] += p[2]
                dv[low] += p[3]
            whole += [torch.cat([p[1] for _, p in parts]), dk.unsqueeze(1), dv.unsqueeze(1)]
        got.append(whole)
    return tuple(torch.cat(t, 1) for t in zip(*got))


def exact(case, seed):
    global own
    kept, own = own, False  # the inputs need no library
    try:
        state = prepare(case, seed)
    finally:
        own = kept
    do = case["do"]
    if do.startswith("attention"):
        got, at = [], _offsets(_tokens_of(case))
        for a, b in zip(at, at[1:]):
            where = torch.arange(b - a, device=_DEVICE)
            dout = state["dout"][a:b] if do == "attention_train" else None
            if b > a:
                got.append(_exact_heads(state, slice(a, b), state["k"][a:b], state["v"][a:b], where, where, dout))
        out = tuple(torch.cat(t) for t in zip(*got))
        return out if do == "attention_train" else out[0]
    if do in ("step", "chunk"):
        got, sinks, window = [], case["sinks"], case["window"]
        cache_k, cache_v = state["cache_k"].clone(), state["cache_v"].clone()
        new = [1] * case["sequences"] if do == "step" else _tokens_of(case)
        at = _offsets(new)
        for i, (a, b, past) in enumerate(zip(at, at[1:], _past_of(case))):
            if a == b:
                continue
            # what the cache still holds of the past, and the new tokens behind it
            key = [p for p in range(past) if p < sinks or p >= past - window]
            slot = [p if p < sinks else sinks + (p - sinks) % window for p in key]
            slot, key = _lengths(slot, torch.int64), _lengths(key + list(range(past, past + b - a)), torch.int64)
            keys = torch.cat([state["cache_k"][i][:, slot].transpose(0, 1), state["k"][a:b]])
            values = torch.cat([state["cache_v"][i][:, slot].transpose(0, 1), state["v"][a:b]])
            where = torch.arange(past, past + b - a, device=_DEVICE)
            got.append(_exact_heads(state, slice(a, b), keys, values, where, key)[0])
            for p in range(past, past + b - a):
                s = p if p < sinks else sinks + (p - sinks) % window
                cache_k[i, :, s], cache_v[i, :, s] = state["k"][a + p - past], state["v"][a + p - past]
        return torch.cat(got), cache_k, cache_v
    kind = _TYPE[case["type"]]
    # h is an output of its own, rounded, and what is normed
    h = (state["x"].double() + state["residual"].double()).to(kind).double()
    gain = state["gain"].double()
    rms = torch.sqrt(h.square().sum(1, keepdim=True) / case["cols"] + EPS)
    y = h / rms * gain
    if do == "norm":
        return y, h
    if do == "norm_linear8":
        return _nearest_fp8(y) @ _fp4_values(state["codes"], state["scales"], case["cols"], torch.float64).T.contiguous(), h
    dy = state["dy"].double()
    along = (dy * gain * h).sum(1, keepdim=True) / case["cols"]
    dx = state["dh"].double() + dy * gain / rms - h * along / rms ** 3
    return y, h, dx, dx, (dy * h / rms).sum(0)
