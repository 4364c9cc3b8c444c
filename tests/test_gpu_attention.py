"""Attention, its gradients and its cache against the oracle's 64-bit definitions.

Tolerances, with u half a step of the type (2^-8, 2^-11, 2^-24 of the value) and e = 2^-24:

* a score is a sum of `dim` products in 32 bits: off by es = 2 (dim + 8) e sum |q k|, times
  the scale in its exponent;
* a weight is exp2 of a rounded multiply-add, within a few e of the exponent's size: its
  relative error is w = es + 8 e (|s| + 4), where |s| is the largest score of the row; the
  same again for the sum that divides it, whose own additions take n e;
* weights are rounded to the type before they are multiplied: u, or in float16 2^-32 of the
  largest for those too small for that; sums over n keys: 2 (n + 8) e;
* the output is rounded: u of it;
* exp2 gives zero for what is below 2^-126, the smallest normal number of 32 bits, and the
  matrix instructions may take operands below that as zero: weights, and ds, may be off by so
  much (a first run had counted only relative errors, and a weight of 2^-125 in a sum alone).

Gradients: lse is stored in 32 bits, so p is off by w and 8 e (|lse| + 4) more; dp and
delta = dout . out are sums in 32 bits, but out has been rounded, so delta is off by u sum
|dout out| besides; p and ds are rounded to the type (float16's ds times a power of two: 2^-36
of the largest in its sum for the small ones); sums over n rows.
"""

import math

import numpy as np
import pytest

from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2401_14351_amd import binding, operators as op  # noqa: E402

TYPES = [torch.bfloat16, torch.float16, torch.float32]
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
E, FLUSH = 2.0 ** -24, 2.0 ** -126


@pytest.fixture(autouse=True)
def _device(gpu_device):
    return gpu_device


def host(t):
    return t.detach().double().cpu().numpy()


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def ids(values, bits=32):
    return torch.tensor(values, dtype=torch.int32 if bits == 32 else torch.int64, device="cuda")


def assert_within(got, want, bound, dtype, what):
    assert got.dtype == dtype
    g = host(got)
    assert g.shape == want.shape, what
    tol = bound + (np.abs(want) + bound) * UNIT[dtype] + SMALLEST[dtype]
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {want[bad][0]}, " \
                          f"allowed {tol[bad][0]}"


def head(q, k, v, seen, scale, dtype, dout=None):
    """Of one head: [(value, bound), ...] of the output, and with dout of dq, dk and dv."""
    u, dim, n = UNIT[dtype], q.shape[1], max(1, int(seen.sum(1).max()))
    # what is not seen counts nowhere
    q_, k_, v_ = (np.where(np.isfinite(t), t, 0.0) for t in (q, k, v))
    out, p, lse = O.attend(q, k, v, seen, scale)
    s = np.where(seen, scale * (q_ @ k_.T), 0.0)
    es = np.where(seen, 2 * (dim + 8) * E * scale * (np.abs(q_) @ np.abs(k_).T), 0.0)
    w = es.max(1, keepdims=True) + 8 * E * (np.abs(s).max(1, keepdims=True) + 4)
    tiny = 2.0 ** -32 if dtype == torch.float16 else 0.0
    rel = u + 2 * w + (n + 2 * (n + 8)) * E
    got = [(out, rel * (p @ np.abs(v_)) + (tiny + FLUSH) * (seen @ np.abs(v_)))]
    if dout is None:
        return got
    o_ = np.where(np.isfinite(dout), dout, 0.0)
    wp = 2 * w + 8 * E * (np.abs(lse)[:, None] + 4) + n * E
    dp = np.where(seen, o_ @ v_.T, 0.0)
    delta = (o_ * out).sum(1, keepdims=True)
    e_dp = 2 * (dim + 8) * E * (np.abs(o_) @ np.abs(v_).T + np.abs(o_) @ np.abs(out).T.max(1, keepdims=True)) + \
        u * (np.abs(o_) * np.abs(out)).sum(1, keepdims=True) + (np.abs(o_) * got[0][1]).sum(1, keepdims=True)
    ds = p * (dp - delta)
    e_ds = np.where(seen, p * e_dp + np.abs(ds) * (u + wp + 8 * E) + FLUSH * (1 + np.abs(dp - delta)), 0.0)
    small = 2.0 ** -36 if dtype == torch.float16 else 0.0
    e_q, e_k = e_ds + small * np.abs(ds).max(1, keepdims=True), e_ds + small * np.abs(ds).max(0, keepdims=True)
    sums = 4 * (max(n, int(seen.sum(0).max())) + 16) * E
    dq, dk, dv = O.attend_grad(dout, q, k, v, seen, scale)
    got.append((dq, scale * (e_q @ np.abs(k_) + sums * (np.abs(ds) @ np.abs(k_)))))
    got.append((dk, scale * (e_k.T @ np.abs(q_) + sums * (np.abs(ds).T @ np.abs(q_)))))
    got.append((dv, ((u + wp + sums) * p).T @ np.abs(o_) + (2.0 ** -40 * (dtype == torch.float16) + FLUSH) * (seen.T @ np.abs(o_))))
    return got


def expect(q, k, v, lengths, window, sinks, scale, dtype, dout=None, past=None):
    """[(value, bound), ...] of packed sequences; rows of no sequence are zeros."""
    group = q.shape[1] // k.shape[1]
    shapes = [q.shape] + ([q.shape, k.shape, v.shape] if dout is not None else [])
    want = [(np.zeros(s), np.zeros(s)) for s in shapes]
    at = 0
    for n in lengths:
        seen = O.visible(range(n), range(n), window, sinks)
        rows = slice(at, at + n)
        at += n
        if not n:
            continue
        for h in range(q.shape[1]):
            kv = h // group
            got = head(q[rows, h], k[rows, kv], v[rows, kv], seen, scale, dtype, None if dout is None else dout[rows, h])
            for i, (value, bound) in enumerate(got):
                to = h if i < 2 else kv
                want[i][0][rows, to] += value
                want[i][1][rows, to] += bound
    return want


def check(q, k, v, lengths, window, sinks, dtype, scale=None, offsets=None, dout=None, pad=0):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    if offsets is None and (len(lengths) > 1 or pad):
        offsets = ids(np.concatenate([[0], np.cumsum(lengths)]))
    if dout is None:
        out = op.attention(q, k, v, window=window, sinks=sinks, offsets=offsets, scale=scale)
        got = [out]
    else:
        leaves = [t.detach().requires_grad_() for t in (q, k, v)]
        out = op.attention(*leaves, window=window, sinks=sinks, offsets=offsets, scale=scale)
        got = [out, *torch.autograd.grad(out, leaves, dout)]
    want = expect(host(q), host(k), host(v), lengths, window, sinks, scale, dtype, None if dout is None else host(dout))
    for name, g, (value, bound) in zip(("out", "dq", "dk", "dv"), got, want):
        assert_within(g, value, bound, dtype, name)


# lengths, heads, key/value heads, elements, window, sinks
CASES = [
    ([1], 1, 1, 1, None, 0), ([1], 8, 2, 64, 1, 0), ([2, 1], 2, 1, 16, None, 0), ([31], 3, 3, 37, None, 0), ([32], 2, 2, 64, 1, 0),
    ([33, 64], 2, 1, 64, 8, 0), ([65], 2, 2, 128, None, 0), ([127], 1, 1, 128, 64, 1), ([128], 2, 1, 96, 63, 4),
    ([129, 1, 0, 30], 2, 2, 80, 65, 2), ([5, 0, 7], 4, 1, 8, 3, 1), ([0, 0, 3], 2, 2, 24, None, 0), ([200], 3, 1, 65, 2, 70),
    ([150], 2, 1, 128, 30, 140), ([300], 2, 2, 64, 128, 0), ([260, 70], 6, 2, 127, 100, 3), ([40], 16, 1, 128, 17, 5),
    ([64, 64], 5, 1, 33, 64, 64), ([257], 1, 1, 72, None, 9), ([3] * 70, 2, 1, 32, 2, 0), ([400], 1, 1, 128, 40, 4),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_and_gradients(case, dtype):
    lengths, heads, kv, dim, window, sinks = CASES[case]
    n = sum(lengths)
    q, k, v = (normal((n, h, dim), dtype, 10 * case + i) for i, h in enumerate((heads, kv, kv)))
    check(q, k, v, lengths, window, sinks, dtype, dout=normal((n, heads, dim), dtype, 10 * case + 3, 0.1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,kv,dim,window,sinks", [([900], 4, 1, 64, 50, 3), ([700, 1, 0, 300], 3, 3, 40, 20, 1),
                                                               ([400, 500], 2, 1, 128, 10, 200), ([60] * 10, 2, 2, 64, 7, 100),
                                                               ([5] * 66 + [300], 2, 2, 33, 4, 129), ([1500], 1, 1, 80, 1, 2)])
def test_sinks_far_behind_the_window(lengths, heads, kv, dim, window, sinks, dtype):
    """Gradients of sinks, which rows far behind the window see: summed apart."""
    n = sum(lengths)
    q, k, v = (normal((n, h, dim), dtype, i) for i, h in enumerate((heads, kv, kv)))
    check(q, k, v, lengths, window, sinks, dtype, dout=normal((n, heads, dim), dtype, 3, 0.1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("std,scale", [(8.0, 1.0), (30.0, 0.125), (1e-3, 1.0), (1.0, 1e-30), (1.0, 40.0)])
def test_scores_of_any_size(dtype, std, scale):
    """Rows that one key dominates, that all share alike, and running maxima that grow a lot."""
    q, k, v = (normal((190, 2, 64), dtype, i, std) for i in range(3))
    check(q, k, v, [190], None, 0, dtype, scale=scale, dout=normal((190, 2, 64), dtype, 4))


@pytest.mark.parametrize("std", [1e-7, 1e-6, 1e-4, 1.0, 100.0, 1000.0])
@pytest.mark.parametrize("v_std", [1e-3, 1.0, 30.0])
def test_half_gradients_of_any_size(std, v_std):
    """float16: gradients near its smallest and largest numbers."""
    q, k = normal((150, 4, 64), torch.float16, 1), normal((150, 2, 64), torch.float16, 2)
    v = normal((150, 2, 64), torch.float16, 3, v_std)
    dout = normal((150, 4, 64), torch.float16, 4, std)
    want = expect(host(q), host(k), host(v), [150], 70, 2, 0.125, torch.float16, host(dout))
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = op.attention(*leaves, window=70, sinks=2, scale=0.125)
    for g, (value, bound), name in zip(torch.autograd.grad(out, leaves, dout), want[1:], ("dq", "dk", "dv")):
        fits = np.abs(value) + bound < 65504
        got = host(g)
        assert np.isfinite(got[fits]).all(), name
        tol = bound + (np.abs(value) + bound) * 2.0 ** -11 + 2.0 ** -25
        assert (np.abs(got - value) <= tol)[fits].all(), name


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_equal_halves(dtype):
    """Gradients whose rows come from different sizes: one row's are not lost beside another's."""
    q, k, v = (normal((140, 1, 64), dtype, i) for i in range(3))
    dout = normal((140, 1, 64), dtype, 5) * torch.logspace(-3, 2, 140, device="cuda").view(-1, 1, 1)
    check(q, k, v, [140], None, 0, dtype, dout=dout.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_that_sees_one_key(dtype):
    """Its output is that key's value and its score's gradient zero, exactly.  Its weight in the
    backward pass is one to within 8 e (|lse| + 4) + es, below 2^-15 for scores under 16."""
    q, k, v, dout = (normal((50, 2, 96), dtype, i) for i in range(4))
    leaves = [t.requires_grad_() for t in (q, k, v)]
    out = op.attention(*leaves, window=1)
    dq, dk, dv = torch.autograd.grad(out, leaves, dout)
    assert torch.equal(out, v) and not dq.any() and not dk.any()
    assert ((dv - dout).abs() <= 2.0 ** -15 * dout.abs()).all() if dtype == torch.float32 else torch.equal(dv, dout)


# ---- layouts ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 80, 31, 128])
def test_strides(dtype, dim):
    """Slices of stacked rows, heads outermost, and rows that start anywhere."""
    n, heads, kv = 100, 4, 2
    stacked = normal((n, heads + 2 * kv, dim), dtype, 1)
    q, k, v = stacked.split([heads, kv, kv], 1)
    check(q, k, v, [60, 40], 33, 2, dtype, dout=normal((n, heads, dim), dtype, 2))
    out = torch.full((n, heads + 3, dim), 7.0, dtype=dtype, device="cuda")
    want = op.attention(q.contiguous(), k.contiguous(), v.contiguous(), window=33)
    assert op.attention(q, k, v, window=33, out=out[:, 1:1 + heads]).data_ptr() == out[:, 1:].data_ptr()
    assert torch.equal(out[:, 1:1 + heads], want) and (out[:, 0] == 7).all() and (out[:, 1 + heads:] == 7).all()
    outer = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(op.attention(*outer, window=33), want)
    flat = torch.empty(n * (heads * (dim + 3)) + 8, dtype=dtype, device="cuda")
    odd = flat[1:1 + n * heads * (dim + 3)].view(n, heads, dim + 3)[..., :dim]
    odd.copy_(q)
    check(odd, k, v, [n], 33, 0, dtype)  # (not the same bytes: a product may be rounded to 32 bits before it is to 16)


@pytest.mark.parametrize("dtype", TYPES)
def test_padding(dtype):
    """Tokens of no sequence, before the first and behind the last: zeros, whatever they hold."""
    n, pad = 150, 300
    q, k, v = (normal((pad, h, 64), dtype, i) for i, h in enumerate((4, 2, 2)))
    dout = normal((pad, 4, 64), dtype, 5)
    for t in (q, k, v, dout):
        t[:20] = math.nan
        t[20 + n:] = math.inf
    want = expect(*(host(t[20:20 + n]) for t in (q, k, v)), [100, 50], 40, 2, 0.125, dtype, host(dout[20:20 + n]))
    for bits in (32, 64):
        leaves = [t.detach().requires_grad_() for t in (q, k, v)]
        out = op.attention(*leaves, window=40, sinks=2, offsets=ids([20, 120, 170], bits))
        for name, g, (value, bound) in zip(("out", "dq", "dk", "dv"), (out, *torch.autograd.grad(out, leaves, dout)), want):
            assert not g[:20].any() and not g[170:].any()
            assert_within(g[20:170], value, bound, dtype, name)
    none = op.attention(q, k, v, offsets=ids([0]))
    assert not none.any()


def test_offsets_that_go_back_or_out():
    """Are taken as the nearest that do not; 70 sequences, so that a wave reads twice."""
    q, k, v = (normal((300, h, 64), torch.bfloat16, i) for i, h in enumerate((2, 1, 1)))
    at = list(range(0, 280, 4))
    wild = at[:30] + [5, -3, at[32], 1 << 40, 250] + at[35:]
    taken = np.minimum(np.maximum.accumulate(np.maximum(wild, 0)), 300)
    want = op.attention(q, k, v, offsets=ids(taken, 64))
    assert torch.equal(op.attention(q, k, v, offsets=ids(wild, 64)), want)
    assert torch.equal(op.attention(q, k, v, offsets=ids([-5, 300])), op.attention(q, k, v))
    assert torch.equal(op.attention(q, k, v, offsets=ids([0, 500])), op.attention(q, k, v))


# ---- what is not seen -------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 3)])
def test_what_is_not_seen_does_not_count(dtype, bad, window, sinks):
    n, heads, kv, dim = 150, 4, 2, 64
    q, k, v = (normal((n, h, dim), dtype, i) for i, h in enumerate((heads, kv, kv)))
    dout = normal((n, heads, dim), dtype, 4)

    def run(q, k, v, dout):
        leaves = [t.detach().requires_grad_() for t in (q, k, v)]
        out = op.attention(*leaves, window=window, sinks=sinks)
        return (out.detach(), *torch.autograd.grad(out, leaves, dout))

    clean = run(q, k, v, dout)
    at = 70
    later = [i for i in range(n) if i >= at and (window is None or i - at < window)]  # who sees it
    others = [i for i in range(n) if i not in later]
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at, :, 5] = bad, bad
    got = run(q, k2, v2, dout)
    for i in (0, 1):
        assert torch.equal(got[i][others], clean[i][others])
    assert not torch.isfinite(got[0][later][:, :, 5]).any()
    # a value alone: those who see it get it, in its column
    got = run(q, k, v2, dout)
    assert torch.equal(got[0][others], clean[0][others]) and torch.equal(got[0][..., :5], clean[0][..., :5])
    assert (got[0][later][..., 5].isnan() if math.isnan(bad) else got[0][later][..., 5] == bad).all()
    # a query's row and its gradient reach the keys that it sees, no others
    q2, d2 = q.clone(), dout.clone()
    q2[at], d2[at, :, 7] = bad, bad
    got = run(q2, k, v, d2)
    hidden = [j for j in range(n) if j > at or (window is not None and at - j >= window and j >= sinks)]
    rest = [i for i in range(n) if i != at]
    assert torch.equal(got[0][rest], clean[0][rest]) and torch.equal(got[1][rest], clean[1][rest])
    for i in (2, 3):
        assert torch.equal(got[i][hidden], clean[i][hidden])


# ---- the cache --------------------------------------------------------------

def held(cache, s, n):
    """What a cache must hold of a sequence: {slot: position}."""
    return {O.slot(p, cache.window, cache.sinks): p for p in range(n)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv,dim,window,sinks", [(4, 2, 64, 16, 3), (2, 2, 128, 1, 0), (20, 1, 40, 50, 0), (6, 2, 33, 300, 2),
                                                       (8, 1, 128, 33, 70), (3, 3, 80, 7, 1), (1, 1, 1, 5, 2)])
def test_cache(heads, kv, dim, window, sinks, dtype):
    """Sequences that grow by chunks of all sizes and by single tokens, round the window many times."""
    pieces = [[5, 0, 40], [1, 1, 1], [90, 3, 0], [1, 1, 1], [1, 1, 1], [0, 130, 2], [1, 1, 1], [2, 17, 64], [1, 1, 1]]
    total = np.sum(pieces, 0)
    seqs = [[normal((int(n), h, dim), dtype, 10 * s + i) for i, h in enumerate((heads, kv, kv))] for s, n in enumerate(total)]
    want = [expect(*(host(t) for t in seq), [len(seq[0])], window, sinks, dim ** -0.5, dtype)[0] for seq in seqs]
    cache = op.KvCache.empty(3, kv, dim, window, sinks, dtype=dtype, device="cuda")
    for t in (cache.k, cache.v):
        t.fill_(math.nan)  # nothing that has not been written is read
    had = np.zeros(3, int)
    for step, new in enumerate(pieces):
        q, k, v = (torch.cat([seqs[s][i][had[s]:had[s] + n] for s, n in enumerate(new)]) for i in range(3))
        lengths = ids(had, 64 if step % 2 else 32)
        single = new == [1, 1, 1]
        offsets = None if single and step % 4 == 1 else ids(np.concatenate([[0], np.cumsum(new)]))
        out = op.attention_cached(q, k, v, cache, lengths, offsets=offsets)
        assert torch.equal(lengths.cpu(), torch.tensor(had, dtype=lengths.dtype))
        at = 0
        for s, n in enumerate(new):
            rows = slice(had[s], had[s] + n)
            assert_within(out[at:at + n], want[s][0][rows], want[s][1][rows], dtype, f"step {step}, sequence {s}")
            at += n
            had[s] += n
            slots = held(cache, s, had[s])
            for c, t in ((cache.k, seqs[s][1]), (cache.v, seqs[s][2])):
                assert torch.equal(c[s][:, list(slots)].transpose(0, 1), t[list(slots.values())])
                free = [i for i in range(window + sinks) if i not in slots]
                assert c[s][:, free].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("past", [0, 1, 255, 256, 1999, 2000, 2003, 2004, 5000])
def test_step_over_a_long_cache(dtype, past):
    """Split over workgroups: the runs' borders, a window filling and full."""
    heads, kv, dim, window, sinks = 6, 2, 64, 2000, 4
    q, k, v = (normal((2, h, dim), dtype, i) for i, h in enumerate((heads, kv, kv)))
    cache = op.KvCache(normal((2, kv, window + sinks, dim), dtype, 4), normal((2, kv, window + sinks, dim), dtype, 5), window, sinks)
    pasts = [past, max(0, past - 700)]
    keep = [cache.k.clone(), cache.v.clone()]
    out = op.attention_cached(q, k, v, cache, ids(pasts))
    for s, p in enumerate(pasts):
        old = [i for i in range(p) if i < sinks or i > p - window]
        slots = [O.slot(i, window, sinks) for i in old]
        for h in range(heads):
            kk, vv = (np.concatenate([host(c[s, h // 3, slots]), host(t[s, h // 3])[None]]) for c, t in zip(keep, (k, v)))
            value, bound = head(host(q[s, h])[None], kk, vv, np.ones((1, len(kk)), bool), dim ** -0.5, dtype)[0]
            assert_within(out[s, h][None], value, bound, dtype, f"sequence {s}, head {h}")
        for c, t, was in ((cache.k, k, keep[0]), (cache.v, v, keep[1])):
            was[s, :, O.slot(p, window, sinks)] = t[s]
            assert torch.equal(c[s], was[s])


@pytest.mark.parametrize("dtype", TYPES)
def test_positions_past_32_bits(dtype):
    """A sequence that has gone on for long is as one that stands at the same slot of the window."""
    q, k, v = (normal((5, h, 64), dtype, i) for i, h in enumerate((4, 2, 2)))
    window, sinks = 37, 3
    base = [normal((1, 2, window + sinks, 64), dtype, i) for i in (5, 6)]
    near = sinks + 5 * window + 11
    far = near + window * ((1 << 40) // window)
    for n, offsets in ((1, None), (5, ids([0, 5]))):
        outs = []
        for past in (near, far):
            cache = op.KvCache(base[0].clone(), base[1].clone(), window, sinks)
            outs.append((op.attention_cached(q[:n], k[:n], v[:n], cache, ids([past], 64), offsets=offsets), cache.k, cache.v))
        for a, b in zip(*outs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [40, 3000])
def test_sequences_that_take_no_part(dtype, window):
    """Their rows are zeros and their cache stays, whatever it and the rows hold."""
    cache = op.KvCache(normal((4, 2, window + 1, 64), dtype, 1), normal((4, 2, window + 1, 64), dtype, 2), window, 1)
    cache.k[1], cache.v[3] = math.nan, math.inf
    q, k, v = (normal((4, h, 64), dtype, i) for i, h in enumerate((4, 2, 2)))
    q[1], k[3] = math.inf, math.nan
    for offsets in (None, ids([0, 1, 2, 3, 4])):
        alone = [op.KvCache(cache.k.clone()[s:s + 1], cache.v.clone()[s:s + 1], window, 1) for s in range(4)]
        c = op.KvCache(cache.k.clone(), cache.v.clone(), window, 1)
        out = op.attention_cached(q, k, v, c, ids([30, -1, 90, -(1 << 31)]), offsets=offsets)
        assert not out[1].any() and not out[3].any()
        for s, past in ((0, 30), (2, 90)):
            want = op.attention_cached(q[s:s + 1], k[s:s + 1], v[s:s + 1], alone[s], ids([past]), offsets=None if offsets is None else ids([0, 1]))
            u = UNIT[dtype]
            assert (out[s] - want[0]).abs().max() <= 8 * u * want[0].abs().max()
            assert torch.equal(c.k[s], alone[s].k[0]) and torch.equal(c.v[s], alone[s].v[0])
        for s in (1, 3):
            for got, was in ((c.k, cache.k), (c.v, cache.v)):
                assert torch.equal(got[s].nan_to_num(3, 4, 5), was[s].nan_to_num(3, 4, 5))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_cache_with_what_is_not_seen(dtype):
    """A slot whose position the window has left, and a new token that earlier ones do not see."""
    window, sinks = 30, 2
    cache = [normal((1, 2, window + sinks, 64), dtype, i) for i in (1, 2)]
    q, k, v = (normal((20, h, 64), dtype, i) for i, h in enumerate((4, 2, 2)))
    past = 100
    clean = op.attention_cached(q, k, v, op.KvCache(cache[0].clone(), cache[1].clone(), window, sinks), ids([past]), offsets=ids([0, 20]))
    bad_k, bad_v, k2, v2 = cache[0].clone(), cache[1].clone(), k.clone(), v.clone()
    first = O.slot(past - window + 5, window, sinks)  # seen by the first five tokens alone
    bad_k[:, :, first] = bad_v[:, :, first] = math.nan
    k2[15] = v2[15] = math.inf
    got = op.attention_cached(q, k2, v2, op.KvCache(bad_k, bad_v, window, sinks), ids([past]), offsets=ids([0, 20]))
    assert torch.equal(got[5:15], clean[5:15]) and got[:5].isnan().all() and not torch.isfinite(got[15:]).any()
    # a token's own slot holds the position that has just left the window
    for long in (30, 2000):
        c = [normal((1, 2, long, 64), dtype, i) for i in (3, 4)]
        one = op.attention_cached(q[:1], k[:1], v[:1], op.KvCache(c[0].clone(), c[1].clone(), long), ids([3 * long + 7]))
        c[0][:, :, 7] = c[1][:, :, 7] = math.nan
        assert torch.equal(op.attention_cached(q[:1], k[:1], v[:1], op.KvCache(c[0], c[1], long), ids([3 * long + 7])), one)


# ---- calls ------------------------------------------------------------------

def test_empty():
    for shape in ((0, 4, 64), (3, 0, 64), (3, 4, 0)):
        t = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        kv = t if shape[1] == 0 else t[:, :2]
        assert op.attention(t, kv, kv).shape == t.shape
    leaf = torch.empty(0, 4, 64, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(op.attention(leaf, leaf, leaf).sum(), leaf)
    assert g.shape == leaf.shape
    c = op.KvCache.empty(0, 2, 64, 8, device="cuda")
    e = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    assert op.attention_cached(e, e, e, c, ids([])).shape == (0, 2, 64)


def test_refusals():
    q = normal((8, 4, 64), torch.bfloat16, 1)
    k = normal((8, 2, 64), torch.bfloat16, 2)
    for args in ((q, k, k[:7]), (q, k.float(), k), (q[0], k, k), (q, k[:, :0], k[:, :0]), (q[:, :3], k, k), (q[..., ::2], k[..., ::2], k[..., ::2]),
                 (q.cpu(), k, k), (q.int(), k.int(), k.int()), (q.expand(8, 4, 64)[:1].expand(8, 4, 64), k, k)):
        with pytest.raises((ValueError, binding.SllmError)):
            op.attention(*args)
    for more in ({"window": 0}, {"window": -1}, {"sinks": -1}, {"scale": 0.0}, {"scale": -1.0}, {"offsets": ids([[0, 8]])}, {"offsets": ids([])},
                 {"offsets": ids([0, 8]).float()}, {"offsets": ids([0, 8]).cpu()}, {"out": q}, {"out": q.float()}, {"out": torch.empty_like(q)[:7]}):
        with pytest.raises((ValueError, binding.SllmError)):
            op.attention(q, k, k, **more)
    with pytest.raises(ValueError):  # writes to a given tensor
        op.attention(q.clone().requires_grad_(), k, k, out=torch.empty_like(q))
    c = op.KvCache.empty(8, 2, 64, 8, device="cuda")
    with pytest.raises(ValueError):
        op.attention_cached(q.clone().requires_grad_(), k, k, c, ids([0] * 8))
    for lengths, offsets in ((ids([0] * 7), None), (ids([0] * 8), ids([0] * 8)), (ids([0] * 8).float(), None)):
        with pytest.raises((ValueError, binding.SllmError)):
            op.attention_cached(q, k, k, c, lengths, offsets=offsets)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError):
            op.attention(torch.autograd.forward_ad.make_dual(q, q), k, k)


def test_same_bytes_every_time():
    q, k, v = (normal((3000, h, 128), torch.bfloat16, i) for i, h in enumerate((8, 2, 2)))
    dout = normal((3000, 8, 128), torch.bfloat16, 4)
    runs = []
    for _ in range(3):
        leaves = [t.detach().requires_grad_() for t in (q, k, v)]
        out = op.attention(*leaves, window=500, sinks=4)
        runs.append((out.detach(), *torch.autograd.grad(out, leaves, dout)))
    for run in runs[1:]:
        for a, b in zip(run, runs[0]):
            assert torch.equal(a, b)


def test_streams():
    """On a stream of its own, beside other calls."""
    q, k, v = (normal((600, h, 64), torch.float16, i) for i, h in enumerate((4, 2, 2)))
    want = op.attention(q, k, v, window=100)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [op.attention(q, k, v, window=100, stream=s) for s in streams for _ in range(3)]
    cache = op.KvCache(normal((2, 2, 2000, 64), torch.float16, 5), normal((2, 2, 2000, 64), torch.float16, 6), 2000)
    torch.cuda.synchronize()
    steps = [op.attention_cached(q[:2], k[:2], v[:2], cache, ids([1500, 1800]), stream=streams[0]) for _ in range(2)]
    for s in streams:
        s.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    torch.cuda.synchronize()
    assert torch.equal(steps[0], steps[1])
    assert torch.equal(steps[0], op.attention_cached(q[:2], k[:2], v[:2], cache, ids([1500, 1800])))


@pytest.mark.parametrize("window", [50, 3000])
def test_a_captured_step_follows_the_lengths(window):
    """A graph of a step and a chunk, replayed with lengths and inputs that the program changes in between."""
    q, k, v = (normal((3, h, 64), torch.bfloat16, i) for i, h in enumerate((4, 2, 2)))
    cache = op.KvCache(normal((3, 2, window + 2, 64), torch.bfloat16, 5), normal((3, 2, window + 2, 64), torch.bfloat16, 6), window, 2)
    eager = op.KvCache(cache.k.clone(), cache.v.clone(), window, 2)
    lengths, offsets = ids([10, 500, 3]), ids([0, 1, 1, 3])
    op.attention_cached(q, k, v, op.KvCache(cache.k.clone(), cache.v.clone(), window, 2), lengths)  # first calls load code
    op.attention_cached(q, k, v, op.KvCache(cache.k.clone(), cache.v.clone(), window, 2), lengths, offsets=offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = op.attention_cached(q, k, v, cache, lengths)
        lengths += 1
        some = op.attention_cached(q, k, v, cache, lengths, offsets=offsets)
    state = torch.tensor([10, 500, 3], dtype=torch.int32, device="cuda")
    for step in range(4):
        q.copy_(normal(q.shape, torch.bfloat16, 20 + step))
        graph.replay()
        want = op.attention_cached(q, k, v, eager, state)
        state += 1
        more = op.attention_cached(q, k, v, eager, state, offsets=offsets)
        torch.cuda.synchronize()
        assert torch.equal(one, want) and torch.equal(some, more)
        assert torch.equal(cache.k, eager.k) and torch.equal(cache.v, eager.v) and torch.equal(lengths, state)
        offsets.copy_(ids([0, 2, 2, 3] if step % 2 == 0 else [0, 0, 3, 3]))


def test_captured_forward_and_gradient_calls():
    """The attention and the gradient's entry point in a graph, each replay as the eager call."""
    q, k, v, dout = (normal((300, h, 64), torch.bfloat16, i) for i, h in enumerate((4, 2, 2, 4)))
    L = binding.lib()

    def run(out, lse, grads, ws):
        stream = torch.cuda.current_stream().cuda_stream
        rows = [op._heads(t, "t") for t in (q, k, v)]
        binding.check(L.sllm_attention(*rows, None, 100, 2, 0.125, op._heads(out, "out"), lse.data_ptr(), 0, stream))
        binding.check(L.sllm_attention_grad(op._heads(dout, "dout"), *rows, op._heads(out, "out"), lse.data_ptr(), None, 100, 2, 0.125,
                                            *(op._heads(g, "g") for g in grads), ws.data_ptr(), ws.numel(), 0, stream))

    def room():
        n = op._workspace(L.sllm_attention_grad_workspace, op._heads(q, "q"), op._heads(k, "k"), None, 100, 2)
        return (torch.empty_like(q), torch.empty(300, 4, device="cuda"), [torch.empty_like(t) for t in (q, k, v)],
                torch.empty(n, dtype=torch.uint8, device="cuda"))

    eager, held_ = room(), room()
    run(*held_)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*held_)
    for step in range(3):
        q.copy_(normal(q.shape, torch.bfloat16, 30 + step))
        graph.replay()
        run(*eager)
        torch.cuda.synchronize()
        for a, b in zip((eager[0], eager[1], *eager[2]), (held_[0], held_[1], *held_[2])):
            assert torch.equal(a, b)


def test_autograd():
    """A non-contiguous gradient, one input of three, a change of a saved tensor, double backward."""
    q, k, v = (normal((40, 2, 64), torch.float32, i).requires_grad_() for i in range(3))
    (a,) = torch.autograd.grad(op.attention(q, k, v).sum(), k)
    b = torch.autograd.grad(op.attention(q, k, v), (q, k, v), torch.ones(40, 2, 64, device="cuda"))
    assert torch.equal(a, b[1])
    (c,) = torch.autograd.grad(op.attention(q.detach(), k.detach(), v).sum(), v)
    assert torch.equal(c, b[2])
    out = op.attention(q, k, v)
    with torch.no_grad():
        k += 1
    with pytest.raises(RuntimeError):
        out.sum().backward()
    (g,) = torch.autograd.grad(op.attention(q, k, v).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    cache = op.KvCache(torch.zeros(40, 2, 8, 64, device="cuda"), torch.zeros(40, 2, 8, 64, device="cuda"), 8)
    used = (cache.k * torch.ones(1, device="cuda", requires_grad=True)).sum() + (cache.k * q.sum()).sum()
    with torch.no_grad():
        op.attention_cached(q, k, v, cache, ids([0] * 40))
    with pytest.raises(RuntimeError):  # the cache has been written to since
        used.backward()


def test_no_gradient_under_capture():
    """A captured backward pass is refused where it would begin; the capture goes on."""
    q = normal((20, 2, 64), torch.float32, 1).requires_grad_()
    gain = torch.ones(64, device="cuda", requires_grad=True)
    with torch.no_grad():
        want = op.attention(q, q, q), op.rms_norm(q, gain)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError):
            op.attention(q, q, q)
        with pytest.raises(ValueError):
            op.rms_norm(q, gain)
        with torch.no_grad():
            got = op.attention(q, q, q), op.rms_norm(q, gain)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("length", [-1, -1 << 40, (1 << 62) + 1, (1 << 63) - 2])
def test_sequences_of_no_length_take_no_part(length):
    """One between two others, by chunks and by single tokens: zeros, its cache as it was, the others as without it."""
    q, k, v = (normal((6, h, 64), torch.bfloat16, i) for i, h in enumerate((4, 2, 2)))
    caches = [op.KvCache(normal((3, 2, 24, 64), torch.bfloat16, 5), normal((3, 2, 24, 64), torch.bfloat16, 6), 20, 4) for _ in range(2)]
    before = caches[0].k.clone(), caches[0].v.clone()
    for offsets in (ids([0, 1, 4, 6]), None):
        tokens = 6 if offsets is not None else 3
        out = [op.attention_cached(*(t[:tokens] for t in (q, k, v)), c, torch.tensor([30, n, 7], device="cuda"), offsets=offsets)
               for c, n in zip(caches, (length, 9))]
        mine = slice(1, 4) if offsets is not None else slice(1, 2)
        assert not out[0][mine].any() and out[1][mine].any()
        out[1][mine] = 0
        assert torch.equal(*out)
        for a, b, c in zip((caches[0].k, caches[0].v), (caches[1].k, caches[1].v), before):
            assert torch.equal(a[1], c[1]) and not torch.equal(b[1], c[1])
            assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_summed_inputs_have_gradients_of_their_own():
    """A norm's input and its residual get equal gradients, not one tensor."""
    x, r = (normal((5, 64), torch.float32, i).requires_grad_() for i in (1, 2))
    y, h = op.rms_norm(x, torch.ones(64, device="cuda"), r)
    (y * y + h).sum().backward()
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [17, 20, 29])
@pytest.mark.parametrize("order", ["up", "down", "only", "below"])
def test_scores_far_from_zero(dtype, power, order):
    """Scores of a large power of two, either sign, and something small, which 32 bits hold exactly.

    Exponents are then exact to 2^-16, and what is off is half a step of each weight and of the output."""
    n, heads, kv, dim = 300, 4, 2, 64
    big = 2.0 ** power
    x = normal((n,), torch.float32, 5, 1.0)
    step = max(2.0 ** (power - 23), 2.0 ** -4)
    x = (x / step).round() * step if power < 24 else torch.zeros_like(x)
    third = torch.arange(n, device="cuda") * 3 // n - 1.0  # -1, 0, 1
    sign = {"up": third, "down": -third, "only": torch.ones_like(third), "below": -torch.ones_like(third)}[order]
    q, k, v = (torch.zeros(n, h, dim, device="cuda") for h in (heads, kv, kv))
    q[..., 0], q[..., 1] = 2.0 ** (power // 2), 1
    k[..., 0], k[..., 1] = (sign * 2.0 ** (power - power // 2))[:, None], x[:, None]
    v = normal((n, kv, dim), dtype, 7)
    q, k = q.to(dtype), k.to(dtype)
    scores = (q.double() @ k.double().repeat_interleave(heads // kv, 1).permute(1, 2, 0)[0]).permute(1, 0, 2).cpu()  # heads x rows x keys
    scores = scores.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
    want = (torch.softmax(scores, -1) @ v.double().cpu().repeat_interleave(heads // kv, 1).transpose(0, 1)).transpose(0, 1)
    tol = (3 * UNIT[dtype] + 2.0 ** -14) * v.double().abs().max().item()
    out = op.attention(q, k, v, scale=1.0)
    assert (out.double().cpu() - want).abs().max() <= tol
    cache = op.KvCache.empty(1, kv, dim, 2000, 0, dtype=dtype, device="cuda")
    out = op.attention_cached(q[:-1], k[:-1], v[:-1], cache, ids([0]), offsets=ids([0, n - 1]), scale=1.0)
    assert (out.double().cpu() - want[:-1]).abs().max() <= tol
    out = op.attention_cached(q[-1:], k[-1:], v[-1:], cache, ids([n - 1]), scale=1.0)
    assert (out.double().cpu() - want[-1:]).abs().max() <= tol


@pytest.mark.parametrize("dtype", TYPES[:2])
@pytest.mark.parametrize("lengths,heads,kv,dim,window,sinks", [([2] * 40, 8, 8, 128, None, 0), ([3, 5, 2, 9, 17, 1, 30] * 4, 6, 2, 40, None, 0),
                                                               ([400], 4, 4, 64, 3, 1), ([190, 193], 4, 1, 128, 2, 0), ([900], 8, 1, 80, 5, 2)])
def test_few_keys_have_exact_gradients(lengths, heads, kv, dim, window, sinks, dtype):
    """Where rows see few keys their gradients by queries and keys are off by their own rounding alone.

    That is at most half a step of each and spread evenly below it: at the most 1 / sqrt(3) = 0.577 of half a step of all
    of them in the root mean square, where each is just above a power of two.  Sums in 32 bits, and scores' gradients in
    two parts (2^-16), add a hundredth."""
    n = sum(lengths)
    q, k, v, d = (normal((n, h, dim), dtype, i) for i, h in enumerate((heads, kv, kv, heads)))
    offsets = ids(np.concatenate([[0], np.cumsum(lengths)]))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(op.attention(*leaves, window=window, sinks=sinks, offsets=offsets), leaves, d)
    wide = [t.double().cpu().requires_grad_() for t in (q, k, v)]
    out, at = [], 0
    for m in lengths:
        qs, ks, vs = (t[at:at + m].transpose(0, 1) for t in wide)
        ks, vs = (t.repeat_interleave(heads // kv, 0) for t in (ks, vs))
        i, j = torch.arange(m)[:, None], torch.arange(m)
        seen = (j <= i) & ((i - j < (window or m)) | (j < sinks))
        s = (qs @ ks.transpose(1, 2) * dim ** -0.5).masked_fill(~seen, -math.inf)
        out.append((torch.softmax(s, -1) @ vs).transpose(0, 1))
        at += m
    want = torch.autograd.grad(torch.cat(out), wide, d.double().cpu())
    for g, w in zip(got[:2], want[:2]):
        assert (g.double().cpu() - w).norm() <= 0.587 * UNIT[dtype] * w.norm()
