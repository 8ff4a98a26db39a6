"""Reading and keeping a part of a long context, in float64 and one kv head at a time.

TEST INFRASTRUCTURE ONLY (see oracle/attention.py).  A kv head's cached keys are an array
[L, r] of the values that the attention sees (code * scale for quantised keys).
"""

from __future__ import annotations

import numpy as np


def bf16_outward(x, up: bool) -> np.ndarray:
    """The bf16 number (8 significant bits) at or next above (up) or below x, as float64; values
    beyond the largest bf16 number become infinite."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    unit = np.maximum(e - 8, -133)                   # subnormal bf16 numbers are multiples of 2^-133
    step = np.ldexp(1.0, unit)
    y = (np.ceil if up else np.floor)(np.ldexp(m, e) / step) * step
    top = (2 - 2.0 ** -7) * 2.0 ** 127
    y = np.where(y > top, np.inf, np.where(y < -top, -np.inf, y))
    # towards zero there is always a finite neighbour
    y = np.where(np.isinf(y) & ((y > 0) != up), np.copysign(top, y), y)
    return np.where(np.isfinite(x), y, x)


def block_bounds(k, block: int, quantised: bool = False):
    """(lo, hi) [blocks, r] of keys [L, r]: bounds of blocks of `block` tokens, rounded outward to
    bf16 for quantised keys; an element with a NaN is bounded by -inf and +inf."""
    k = np.asarray(k, dtype=np.float64)
    lo, hi = [], []
    for t in range(0, len(k), block):
        part = k[t:t + block]
        bad = np.isnan(part).any(0)
        clean = np.where(np.isnan(part), 0.0, part)
        lo.append(np.where(bad, -np.inf, clean.min(0)))
        hi.append(np.where(bad, np.inf, clean.max(0)))
    lo, hi = np.array(lo).reshape(-1, k.shape[1]), np.array(hi).reshape(-1, k.shape[1])
    return (bf16_outward(lo, False), bf16_outward(hi, True)) if quantised else (lo, hi)


def block_scores(q, lo, hi) -> np.ndarray:
    """Scores [blocks] of queries q [G, r]: max over G of sum_i max(q_i lo_i, q_i hi_i), +inf where
    a bound or one of the sums is not finite."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.zeros((len(q), len(lo)))
        for i in range(q.shape[1]):                   # elements in order
            s += np.where(q[:, i, None] < 0, q[:, i, None] * lo[None, :, i], q[:, i, None] * hi[None, :, i])
        odd = ~np.isfinite(lo).all(1) | ~np.isfinite(hi).all(1) | ~np.isfinite(s).all(0)
        return np.where(odd, np.inf, s.max(0))


def block_select(scores, n_select: int, n_first: int = 1, n_last: int = 1) -> np.ndarray:
    """Numbers of the chosen blocks, ascending."""
    n = len(scores)
    if n <= n_select:
        return np.arange(n)
    forced = [i for i in range(n) if i < n_first or i >= n - n_last]
    free = sorted((i for i in range(n) if n_first <= i < n - n_last), key=lambda i: (-scores[i], i))
    return np.array(sorted(forced + free[:n_select - len(forced)]))


def attn_weights(q, k, scale: float, n_q: int) -> np.ndarray:
    """Weights [L] of queries q [G, n_q, r] at the last n_q positions of the context."""
    L = len(k)
    w = np.zeros(L)
    for i in range(n_q):
        p = L - n_q + i
        if p < 0:
            continue
        for h in range(len(q)):
            x = scale * (k[:p + 1] @ q[h, i])
            e = np.exp(x - x.max())
            w[:p + 1] += e / e.sum()
    return w


def evict(w, n_keep: int, n_recent: int) -> np.ndarray:
    """Slots whose tokens are in slots 0, 1, .. afterwards, from weights [L]."""
    L = len(w)
    if L <= n_keep:
        return np.arange(L)
    n, want = L - n_recent, n_keep - n_recent
    v = np.where(np.isnan(w[:n]), -np.inf, w[:n])
    nan = np.isnan(w[:n])
    order = sorted(range(n), key=lambda i: (bool(nan[i]), -v[i], i))   # NaN behind -inf
    best = sorted(order[:want])
    out = np.full(n_keep, -1)
    for i in best:
        if i < want:
            out[i] = i
    rest = iter(i for i in best if i >= want)
    for j in range(want):
        if out[j] < 0:
            out[j] = next(rest)
    out[want:] = np.arange(L - n_recent, L)
    return out
