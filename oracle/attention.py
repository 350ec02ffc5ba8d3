"""Attention over a cache of shares, written from its definition: plain numpy on ``uint64`` words, one
row and key at a time where that matters, nothing shared with the GPU path.

Shapes: ``e``, ``a`` [tokens, heads, d] or [tokens, heads, ld]; pools [pages, page, kv heads, ldp]; the
batch as ``q_start``, ``kv_len``, ``table`` (page ids) and an optional ``head_mask`` [tokens, heads].
Results are written into a copy of ``out``, so whatever a call must leave alone shows."""
from __future__ import annotations

import numpy as np

U = np.uint64


def rescale(party, z, bits):
    """floor(z / 2^bits) on the signed word for party 0, -floor(-z / 2^bits) for party 1."""
    z = np.asarray(z, dtype=np.uint64)
    if party == 0:
        return (z.view(np.int64) >> np.int64(bits)).view(np.uint64)
    return U(0) - ((U(0) - z).view(np.int64) >> np.int64(bits)).view(np.uint64)


def rows(q_start, kv_len, n_heads, causal=True, head_mask=None, max_q=None):
    """(sequence, token, head, keys seen) of every row of the batch."""
    for s, kv in enumerate(kv_len):
        new = int(q_start[s + 1]) - int(q_start[s])
        for j in range(new if max_q is None else min(new, max_q)):
            t = int(q_start[s]) + j
            for h in range(n_heads):
                v = max(int(kv) - new + j + 1, 0) if causal else int(kv)
                if head_mask is not None and not head_mask[t, h]:
                    v = 0
                yield s, t, h, v


def cached(pool, table, s, n, kv_head, d):
    """The first n rows of sequence s, key head kv_head, d words each."""
    page = pool.shape[1]
    out = np.zeros((n, d), dtype=np.uint64)
    for j in range(n):
        out[j] = pool[int(table[s, j // page]), j % page, kv_head, :d]
    return out


def cache_write(party, d_0, d_1, b_i, slots, f_pool, x_pool):
    f_pool, x_pool = f_pool.copy(), x_pool.copy()
    for t, slot in enumerate(slots):
        if 0 <= slot < len(f_pool):
            f_pool[slot] = d_0[t] + d_1[t]
            x_pool[slot] = b_i[t] + f_pool[slot] * U(party)
    return f_pool, x_pool


def cache_read(party, f_pool, x_pool, slots, e, a_i):
    e, a_i = e.copy(), a_i.copy()
    for t, slot in enumerate(slots):
        if 0 <= slot < len(f_pool):
            e[t] = f_pool[slot]
            a_i[t] = x_pool[slot] - f_pool[slot] * U(party)
    return e, a_i


def rotate(party, x, positions, cos, sin, n_heads, shift, bits, m=None, interleaved=False):
    t, width = x.shape
    d, half = width // n_heads, cos.shape[1]
    y = rescale(party, x, shift).reshape(t, n_heads, d).copy()
    src = y.copy()
    for i in range(t):
        pos = int(positions[i]) if 0 <= int(positions[i]) < len(cos) else 0
        for j in range(half):
            p, q = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            c, s = cos[pos, j], sin[pos, j]
            y[i, :, p] = rescale(party, src[i, :, p] * c - src[i, :, q] * s, bits)
            y[i, :, q] = rescale(party, src[i, :, q] * c + src[i, :, p] * s, bits)
    y = y.reshape(t, width)
    return y if m is None else y - m


def scores(party, batch, e, a, f_pool, x_pool, table, c, bits, m, out):
    out, group = out.copy(), e.shape[1] // f_pool.shape[2]
    for s, t, h, v in batch:
        x, f = (cached(pool, table, s, v, h // group, e.shape[2]) for pool in (x_pool, f_pool))
        z = c[t, h, :v] + x @ e[t, h] + f @ a[t, h]
        out[t, h, :v] = rescale(party, z, bits) - (U(0) if m is None else m[t, h, :v])
    return out


def weights(party, batch, d_0, d_1, r, r2, bias, bits, m, out, sums):
    out, sums = out.copy(), sums.copy()
    for _, t, h, v in batch:
        u = d_0[t, h, :v] + (U(0) if d_1 is None else d_1[t, h, :v]) + U(bias)
        w = rescale(party, r2[t, h, :v] + U(2) * u * r[t, h, :v] + U(party) * u * u, bits)
        out[t, h, :v] = w - (U(0) if m is None else m[t, h, :v])
        sums[t, h] = np.add.reduce(w, dtype=np.uint64)
    return out, sums


def values(party, batch, e, a, f_pool, x_pool, table, c, bits, m, out):
    out, group, d = out.copy(), e.shape[1] // f_pool.shape[2], c.shape[2]
    for s, t, h, v in batch:
        x, f = (cached(pool, table, s, v, h // group, d) for pool in (x_pool, f_pool))
        z = c[t, h] + e[t, h, :v] @ x + a[t, h, :v] @ f
        out[t, h] = rescale(party, z, bits) - (U(0) if m is None else m[t, h])
    return out
