"""The cache held in 8 bits by its definition, in numpy: fp32 where the definition rounds, 64 bits elsewhere."""
from __future__ import annotations

import numpy as np

BLOCK = 64
LARGEST = np.float32(3.3895313892515355e38)  # of bf16


def finite(x):
    """fp32 numbers that are bf16 numbers; infinities become the largest of these, NaN 0."""
    x = np.where(np.isnan(x), np.float32(0), x.astype(np.float32))
    return np.clip(x, -LARGEST, LARGEST)


def held(rows):
    """[L][Hkv][d] fp32 rows as they came -> the numbers that the cache holds, 64 bits."""
    x = finite(rows)
    out = x.astype(np.float64)
    whole = len(x) // BLOCK * BLOCK
    if whole:
        b = x[:whole].reshape(-1, BLOCK, *x.shape[1:])
        scale = np.maximum(np.abs(b).max(axis=(1, 3), keepdims=True) / np.float32(127), np.float32(2.0 ** -100))
        code = np.clip(np.rint(b / scale), -127, 127)
        assert code.dtype == np.float32 and scale.dtype == np.float32
        out[:whole] = (code.astype(np.float64) * scale).reshape(x[:whole].shape)
    return out


def attend(q, k, v, prev, scale):
    """q [n][Hq][d], k, v [L][Hkv][d], all 64 bits, L = prev + n.  Returns out [n][Hq][d], lse [Hq][n], and what the bounds on a kernel's error need: the mean
    of |v| under the same weights [n][Hq][d], and the largest sum of |q k| scale over a row's keys [Hq][n]."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    out, mean_abs = np.empty_like(q), np.empty_like(q)
    lse, span = np.empty((hq, n)), np.empty((hq, n))
    for h in range(hq):
        g = h // group
        s = q[:, h] @ k[:, g].T * scale
        a = np.abs(q[:, h]) @ np.abs(k[:, g]).T * scale
        seen = np.arange(prev + n)[None, :] <= prev + np.arange(n)[:, None]
        s = np.where(seen, s, -np.inf)
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(-1, keepdims=True)
        lse[h] = (top + np.log(total))[:, 0]
        span[h] = np.where(seen, a, 0).max(-1)
        out[:, h] = p / total @ v[:, g]
        mean_abs[:, h] = p / total @ np.abs(v[:, g])
    return out, lse, mean_abs, span


def bounds(out, lse, mean_abs, span, d, length):
    """What a bf16 kernel's output and log-sum-exp may be off by.

    A logit is a sum of d products of bf16 numbers in fp32, each exact: off by at most (d + 2) 2^-24 times the sum of their magnitudes (the scale's
    rounding and the exponent's subtraction included), call it e, relative to its weight.  Weights are rounded to bf16 for the second product, half a
    step, 2^-8 of each, and their sum is not: 2^-8 of the weighted mean of |v|.  The exponential is good to 2^-22, sums of `length` terms in fp32
    to (64 + length / 64) 2^-24 (64 in a row, then blocks).  The output is rounded once, 2^-8 of it.

    What an exponential gives below fp32's smallest normal number is lost: each key's scale times weight then is less than 2^-126, and its share of the
    output, the sum of weights being at least 1, less than 2^-126 times its code, at most 127 (or its value, where that is held as it came)."""
    e = (d + 2) * 2.0 ** -24 * span + 2.0 ** -22 + (64 + length / 64 + 64) * 2.0 ** -24
    e_out = 2 * e.T[:, :, None] * mean_abs + length * 2.0 ** -119
    return 2.0 ** -8 * (np.abs(out) + mean_abs) * (1 + 2.0 ** -7) + e_out, e + 2.0 ** -22 * (np.abs(lse) + span + 8)
