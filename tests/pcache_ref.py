"""The cache in pages by its definition, in 64 bits, and what a kernel's results may be off by."""
from __future__ import annotations

import numpy as np
import torch

TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def attend(q, k, v, visible, scale):
    """q [n][Hq][d], k, v [L][Hkv][d], visible [n][L]: out [n][Hq][d], lse [Hq][n], the mean of |v| under the same weights, and the largest sum of |q k| scale over
    a row's keys [Hq][n].  Rows that see nothing: zeros and -inf."""
    q, k, v = (t.double().numpy() for t in (q, k, v))
    n, hq, d = q.shape
    group = hq // k.shape[1]
    out, mean_abs, lse, span = np.zeros_like(q), np.zeros_like(q), np.full((hq, n), -np.inf), np.zeros((hq, n))
    if not k.shape[0]:
        return out, lse, mean_abs, span
    some = visible.any(-1)
    for h in range(hq):
        keys, values = k[:, h // group], v[:, h // group]
        s = np.where(visible, q[:, h] @ keys.T * scale, -np.inf)
        top = np.where(some, s.max(-1), 0)
        p = np.exp(s - top[:, None])
        total = np.where(some, p.sum(-1), 1)
        lse[h] = np.where(some, top + np.log(total), -np.inf)
        span[h] = np.where(visible, np.abs(q[:, h]) @ np.abs(keys).T * scale, 0).max(-1)
        out[:, h] = p / total[:, None] @ values
        mean_abs[:, h] = p / total[:, None] @ np.abs(values)
    return out, lse, mean_abs, span


def bounds(out, lse, mean_abs, span, d, length, dtype):
    """What a kernel's output and log-sum-exp may be off by.

    A logit is a sum of d products in fp32, off by at most d half steps, 2^-24, of the sum of their magnitudes, four more with the scale, the subtraction of
    the reference and the reference's own rounding: (d + 4) 2^-24 span, relative to the weight.  An exponential is good to 2^-22; a row's reference moves a few times, a factor
    of such an exponential each: twelve of them together.  Sums of `length` terms in any order, with a rounding for each time that the reference may move (every 16 keys):
    (1.1 length + 16) 2^-24.  That is e, of the weights, their sum and their products with v.  In bf16 the weights are rounded for the second product, half a
    step, 2^-8, and the output once, 2^-8 of it; fp32's output has the division's and the product's half step, 2^-23.  What an exponential gives below fp32's smallest normal
    number is lost: 2^-126 a key of |v|, here at most 2^10."""
    e = (d + 4) * 2.0 ** -24 * span + 12 * 2.0 ** -22 + (1.1 * length + 16) * 2.0 ** -24
    rounding = 2.0 ** -8 * (np.abs(out) + mean_abs) * (1 + 2.0 ** -7) if dtype == "bf16" else 2.0 ** -23 * np.abs(out)
    return rounding + 2 * e.T[:, :, None] * mean_abs + length * 2.0 ** -116, e + 2.0 ** -22 * (np.where(np.isfinite(lse), np.abs(lse), 0) + span + 8)


def assign(lens, new, free, n_free, tables, page, n_slots):
    """kvfold_pcache_assign in plain Python on lists; returns (tables, lens_after, cu_new, slots, positions, n_free_after, status)."""
    tables = [list(r) for r in tables]
    width = len(tables[0]) if tables else 1 << 30
    up = lambda n: -(-n // page)
    status = 8 if any(x < 0 for x in list(lens) + list(new)) else 0
    good = [(p, n) for p, n in zip(lens, new) if p >= 0 and n >= 0]
    count = min(max(n_free, 0), len(free))
    status |= 1 if sum(up(p + n) - up(p) for p, n in good) > count else 0
    status |= 2 if any(up(p + n) > width for p, n in good) else 0
    status |= 4 if sum(n for _, n in good) > n_slots else 0
    if status:
        return tables, list(lens), [0] * (len(lens) + 1), [-1] * n_slots, [-1] * n_slots, n_free, status
    cu, slots, positions = [0], [], []
    for s, (p, n) in enumerate(zip(lens, new)):
        for j in range(up(p), up(p + n)):
            count -= 1
            tables[s][j] = free[count]
        for at in range(p, p + n):
            slots.append(tables[s][at // page] * page + at % page)
            positions.append(at)
        cu.append(cu[-1] + n)
    more = [-1] * (n_slots - len(slots))
    return tables, [p + n for p, n in zip(lens, new)], cu, slots + more, positions + more, count, 0
