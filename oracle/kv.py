"""Float64 oracle of the key-value cache operators (test infrastructure only).

A sequence's cache is given as plain arrays of values: ``k`` and ``v`` of
shape ``[heads, entries, head_dim]``, ``weight`` and ``pos`` ``[heads,
entries]``; pages are the concern of the code under test.
"""
from __future__ import annotations

import numpy as np


def e4m3_values() -> np.ndarray:
    """The 256 numbers of the 8-bit format with 4 exponent and 3 mantissa bits
    (bias 7; no infinity, 0x7f and 0xff are NaN)."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    x = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7), m / 8 * 2.0 ** -6)
    x[(b & 127) == 127] = np.nan
    return np.where(b >> 7, -x, x)


def e4m3_encode(x) -> np.ndarray:
    """Nearest of those numbers, ties to the even pattern, clamped to +-448."""
    x = np.asarray(x, np.float64)
    grid = e4m3_values()[:127]                       # 0 .. 448, ascending
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    code = np.where(up, hi, lo) | (np.signbit(x).astype(np.int64) << 7)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def rotate(x, cos, sin, interleaved=False):
    """Rotary embedding of rows ``x [..., d]`` with the angles' cosines and
    sines ``[..., d / 2]``."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    y = np.empty_like(x)
    for i in range(d // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
        y[..., a] = x[..., a] * cos[..., i] - x[..., b] * sin[..., i]
        y[..., b] = x[..., b] * cos[..., i] + x[..., a] * sin[..., i]
    return y


def attend(q, k, v, scale, start=0):
    """One token: ``q [n_q_heads, d]`` over entries ``start`` on of ``k, v
    [n_kv_heads, n, d]``.  Returns out, lse and every entry's probability
    summed over the query heads of its kv head."""
    hq, hkv, n = q.shape[0], k.shape[0], k.shape[1]
    out = np.zeros((hq, v.shape[2]))
    lse = np.full(hq, -np.inf)
    share = np.zeros((hkv, n))
    for h in range(hq):
        g = h // (hq // hkv)
        s = scale * (k[g, start:] @ q[h])
        if s.size == 0 or np.all(s == -np.inf):
            continue
        with np.errstate(invalid="ignore"):
            top = s.max()
            p = np.exp(s - top)
            lse[h] = top + np.log(p.sum())
            p = p / p.sum()
        out[h] = p @ v[g, start:]
        share[g, start:] += p
    return out, lse, share


def evict_plan(weight, pos, budget, recent):
    """One head of one sequence: (places, sources): entry ``sources[i]`` moves
    to place ``places[i]``."""
    n = len(weight)
    if n <= budget:
        return [], []
    last = int(np.max(pos))

    def rank(i):
        w = float(weight[i])
        if int(pos[i]) > last - recent:
            return (0, 0.0, i)
        return (2, 0.0, i) if np.isnan(w) else (1, -w, i)

    kept = set(sorted(range(n), key=rank)[:budget])
    return [i for i in range(budget) if i not in kept], [i for i in range(budget, n) if i in kept]
