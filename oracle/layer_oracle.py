"""CPU oracle of the operators around a layer's matrices, in 64 bits: norms, MX FP8,
attention and its cache.

TEST INFRASTRUCTURE ONLY, like the other oracles: the plain definitions, sharing nothing
with the product path.  numpy arrays of doubles throughout.
"""

import math

import numpy as np

BLOCK = 32
# E4M3: four bits of exponent, three behind the leading one, no infinities, 0x7f a NaN
E4M3 = np.array([(k & 7) * 2.0 ** -9 if k < 8 else (1 + (k & 7) / 8) * 2.0 ** ((k >> 3) - 7) for k in range(127)])


# ---- MX FP8 -----------------------------------------------------------------

def quantize8(x):
    """(codes, scales) of the matrix x as they are stored."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    codes = np.zeros((rows, blocks * BLOCK), np.uint8)
    scales = np.zeros((rows, -(-blocks // 16) * 16), np.uint8)
    middle = (E4M3[1:] + E4M3[:-1]) / 2
    for r in range(rows):
        for b in range(blocks):
            v = np.zeros(BLOCK)
            part = x[r, b * BLOCK:(b + 1) * BLOCK]
            v[:len(part)] = part
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top, e = np.abs(v).max(), -127
            if top:
                e = max(math.frexp(top)[1] - 9, -127)
                if math.ldexp(448.0, e) < top:
                    e += 1
            scales[r, b] = e + 127
            y = np.ldexp(np.abs(v), -e)
            k = np.searchsorted(middle, y)                # how many middles lie below
            tie = (k < 126) & (middle[np.minimum(k, 125)] == y)
            k = k + (tie & (k % 2 == 1))                  # of two equally near, the even code
            codes[r, b * BLOCK:(b + 1) * BLOCK] = k | (np.signbit(v) << 7)
    return codes, scales


def dequantize8(codes, scales, cols):
    blocks = -(-cols // BLOCK)
    level = np.append(E4M3, np.nan)
    v = np.where(codes & 128, -1.0, 1.0) * level[codes & 127]
    s = scales[:, :blocks].astype(np.float64)
    v = v.reshape(len(codes), blocks, BLOCK) * 2.0 ** (s - 127)[..., None]
    v[s == 255] = np.nan
    return v.reshape(len(codes), -1)[:, :cols]


# ---- norms ------------------------------------------------------------------

def norm(h, gain, eps):
    h = np.asarray(h, np.float64)
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * gain


def norm_grad(dy, dh, h, gain, eps):
    """(dx, dgain): of norm(h) with dy, and of h itself with dh."""
    f = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    s = dy * gain
    return dh + f * (s - h * f * f * (s * h).mean(-1, keepdims=True)), (dy * h * f).sum(0)


# ---- attention --------------------------------------------------------------

def visible(at, key, window, sinks):
    """(queries, keys): who sees whom, by their positions; window None: no window."""
    at, key = np.asarray(at)[:, None], np.asarray(key)[None, :]
    seen = key <= at
    return seen if window is None else seen & ((at - key < window) | (key < sinks))


def attend(q, k, v, seen, scale):
    """One head: (out, weights, lse).  Rows of k and v that a query does not see are not
    looked at."""
    out, weights, lse = np.zeros((len(q), v.shape[1])), np.zeros((len(q), len(k))), np.zeros(len(q))
    for i in range(len(q)):
        j = np.flatnonzero(seen[i])
        s = scale * (k[j] @ q[i])
        top = s.max()
        p = np.exp(s - top)
        lse[i] = top + math.log(p.sum())
        weights[i, j] = p / p.sum()
        out[i] = weights[i, j] @ v[j]
    return out, weights, lse


def attend_grad(dout, q, k, v, seen, scale):
    """(dq, dk, dv) of one head, pair by seen pair."""
    out, p, _ = attend(q, k, v, seen, scale)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for i in range(len(q)):
        j = np.flatnonzero(seen[i])
        ds = p[i, j] * (v[j] @ dout[i] - dout[i] @ out[i])
        dq[i] = scale * (ds @ k[j])
        dk[j] += scale * ds[:, None] * q[i]
        dv[j] += p[i, j][:, None] * dout[i]
    return dq, dk, dv


def slot(p, window, sinks):
    return p if p < sinks else sinks + (p - sinks) % window
