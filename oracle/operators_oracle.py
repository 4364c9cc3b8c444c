"""CPU oracle of the operators on loaded weights, in 64 bits.

TEST INFRASTRUCTURE ONLY, like the loader's oracle: the plain definitions,
sharing nothing with the product path.  numpy arrays of doubles throughout.

MX FP4 follows the OCP Microscaling formats: 32 columns share a power of two
2^(s - 127), elements are E2M1.  Where that leaves a choice: the scale is
2^(floor(log2 of the largest magnitude) - 2), elements round to nearest with
ties to the even code and saturate, the smallest scale serves a block of zeros,
and a block with an infinity or a NaN is NaN throughout (scale 255, codes 0).
"""

import math

import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
BLOCK = 32


def _pitches(cols):
    blocks = -(-cols // BLOCK)
    return blocks, -(-blocks // 16) * 16


def quantize(x):
    """(codes, scales) of the matrix x as they are stored."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks, scale_pitch = _pitches(cols)
    codes = np.zeros((rows, blocks * 16), np.uint8)
    scales = np.zeros((rows, scale_pitch), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            v = np.zeros(BLOCK)
            part = x[r, b * BLOCK:(b + 1) * BLOCK]
            v[:len(part)] = part
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            e = max(math.frexp(top)[1] - 3, -127) if top else -127
            scales[r, b] = e + 127
            # distance to every level; of two equally near, the even code
            d = np.abs(np.abs(v)[:, None] * 2.0 ** -e - LEVELS)
            near = d.argmin(1)
            tie = (near < 7) & (d[np.arange(BLOCK), np.minimum(near + 1, 7)] == d[np.arange(BLOCK), near])
            near = np.where(tie & (near % 2 == 1), near + 1, near)
            code = (near | (np.signbit(v) << 3)).astype(np.uint8)
            codes[r, b * 16:(b + 1) * 16] = code[0::2] | (code[1::2] << 4)
    return codes, scales


def dequantize(codes, scales, cols):
    """What stored codes and scales stand for."""
    blocks, _ = _pitches(cols)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], blocks, BLOCK)
    s = scales[:, :blocks].astype(np.float64)
    v = np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7] * 2.0 ** (s - 127)[..., None]
    v[s == 255] = np.nan
    return v.reshape(codes.shape[0], blocks * BLOCK)[:, :cols]


def linear(x, w):
    return np.asarray(x, np.float64) @ np.asarray(w, np.float64).T


def linear_grad(dy, w):
    return np.asarray(dy, np.float64) @ np.asarray(w, np.float64)


def embedding(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < len(table):
            out[i] = scale * np.asarray(table[v], np.float64)
    return out


def embedding_grad(dy, ids, vocab, scale, grad=None):
    """grad (zeros if none) plus the lookup's gradient."""
    out = np.zeros((vocab, dy.shape[1])) if grad is None else np.array(grad, np.float64)
    for i, v in enumerate(ids):
        if 0 <= v < vocab:
            out[v] += scale * np.asarray(dy[i], np.float64)
    return out
