"""fp64 oracle of the operators between a projection and the attention.

Written from the definitions: one row, one pair, one request at a time where
that keeps it plain.  Test infrastructure only.
"""

import numpy as np


def angles(positions, inv_freq, pair_axis):
    """[B, S, pairs] angles position[axis] * inv_freq, positions [n_axes, B, S] integers."""
    pos = np.asarray(positions, dtype=np.float64)
    return np.stack([pos[a] * np.float64(f) for f, a in zip(inv_freq, pair_axis)], axis=-1) \
        if len(inv_freq) else np.zeros(pos.shape[1:] + (0,))


def pair_index(rot, layout):
    """The two elements of each pair."""
    j = np.arange(rot // 2)
    return (j, j + rot // 2) if layout == "half" else (2 * j, 2 * j + 1)


def rotate(y, theta, rot, layout):
    """y [B, H, S, r] with the pairs of its first rot elements turned by theta [B, S, pairs]."""
    i0, i1 = pair_index(rot, layout)
    c, s = np.cos(theta)[:, None], np.sin(theta)[:, None]
    out = y.copy()
    out[..., i0] = y[..., i0] * c - y[..., i1] * s
    out[..., i1] = y[..., i0] * s + y[..., i1] * c
    return out


def rms(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def norm_rope(x, w, theta, rot, layout, norm=True, eps=1e-6):
    """RMS norm over the last axis (if norm), weight w [r] (offset already added), rotation."""
    y = x * rms(x, eps) * w if norm else x
    return rotate(y, theta, rot, layout)


def norm_rope_backward(x, w, dy, theta, rot, layout, norm=True, eps=1e-6):
    """(dx, dw, sum |terms of dw|, bound of dx's terms) for dL/d(norm_rope) = dy."""
    g = rotate(dy, -theta, rot, layout)
    if not norm:
        return g, None, None, np.abs(dy).max(axis=-1, keepdims=True)
    rho = rms(x, eps)
    xhat = x * rho
    gu = g * w
    mean = np.mean(gu * xhat, axis=-1, keepdims=True)
    dx = rho * (gu - xhat * mean)
    size = rho * (np.abs(w).max() * np.abs(g).max(axis=-1, keepdims=True)
                  + np.abs(xhat) * np.mean(np.abs(gu * xhat), axis=-1, keepdims=True))
    terms = g * xhat
    return dx, terms.sum(axis=(0, 1, 2)), np.abs(terms).sum(axis=(0, 1, 2)), size


def block_tables(seq_lens, new_lens, page_table, free_pages, free_count, page_size, rows, tokens_per_seq):
    """One step of the page pool, request by request.  Returns a dict of the arrays after it."""
    B, max_pages = page_table.shape
    table, stack = page_table.copy(), list(free_pages[:free_count])
    pages_of = lambda n: -(-int(n) // page_size)  # noqa: E731
    for b in range(B):
        if new_lens[b] == -1:
            stack += [int(page_table[b, i]) for i in range(pages_of(seq_lens[b]))]
    top, wanted, needed = len(stack), 0, 0
    lens = np.zeros(B, np.int64)
    offsets = np.zeros(B + 1, np.int64)
    slots = np.full(rows, -1, np.int64)
    positions = np.zeros(rows, np.int64)
    refused = taken = 0
    for b in range(B):
        L, n = int(seq_lens[b]), int(new_lens[b])
        granted = 0
        if n >= 0:
            lens[b] = L
            wanted += n
            ok = L + n <= max_pages * page_size and (n <= tokens_per_seq if tokens_per_seq else wanted <= rows)
            need = pages_of(L + n) - pages_of(L)
            if ok:
                needed += need
                ok = need == 0 or needed <= top
            if ok:
                for i in range(need):
                    table[b, pages_of(L) + i] = stack[top - 1 - taken]
                    taken += 1
                granted, lens[b] = n, L + n
            else:
                refused += 1
        row0 = b * tokens_per_seq if tokens_per_seq else offsets[b]
        for t in range(granted):
            p = L + t
            positions[row0 + t] = p
            slots[row0 + t] = table[b, p // page_size] * page_size + p % page_size
        offsets[b + 1] = offsets[b] + granted
    free = np.array(free_pages, np.int64)
    free[:top - taken] = stack[:top - taken]
    return dict(page_table=table, free_pages=free, free_count=top - taken, seq_lens=lens, offsets=offsets,
                slots=slots, positions=positions, refused=refused)
