"""The paged key/value cache in float64: what an append leaves in it, and the attention over it.

TEST INFRASTRUCTURE ONLY (see the package docstring). Everything is written token by token from the definitions; the
attention of one sequence is :func:`oracle.naive.attention_head` on the keys gathered from its pages.
"""

from __future__ import annotations

import numpy as np

from .naive import attention_head


def rotate(x, angles_cos, angles_sin, begin: int, interleaved: bool):
    """x [..., d] with the dims from ``begin`` on turned: pair number c by the angle whose cosine and sine are
    ``angles_cos[c]``, ``angles_sin[c]``; the pair is (c, c + half) of the turned dims, or (2c, 2c + 1)."""
    y = np.array(x, dtype=np.float64)
    half = len(angles_cos)
    for c in range(half):
        i, j = (begin + 2 * c, begin + 2 * c + 1) if interleaved else (begin + c, begin + half + c)
        y[..., i] = x[..., i] * angles_cos[c] - x[..., j] * angles_sin[c]
        y[..., j] = x[..., j] * angles_cos[c] + x[..., i] * angles_sin[c]
    return y


def token_positions(q_starts, kv_lens):
    """(sequence, position) of every packed token; (-1, -1) for one that belongs to no sequence or would lie
    before position 0."""
    total = int(q_starts[-1])
    out = [(-1, -1)] * total
    for b in range(len(kv_lens)):
        n = int(q_starts[b + 1]) - int(q_starts[b])
        for i in range(n):
            p = int(kv_lens[b]) - n + i
            if p >= 0:
                out[int(q_starts[b]) + i] = (b, p)
    return out


def paged_rows(cache, table_row, n: int, page: int):
    """Keys (or values) 0 .. n-1 of one sequence, [n, H, d], and which of them lie in a page of the cache."""
    pos = np.arange(n)
    pages = np.asarray(table_row)[pos // page] if n else np.zeros(0, dtype=np.int64)
    there = (pages >= 0) & (pages < cache.shape[0])
    rows = cache[np.where(there, pages, 0), :, pos % page, :] if n else np.zeros((0, cache.shape[1], cache.shape[3]))
    return rows, there


def paged_attention(q, k_cache, v_cache, table, kv_lens, q_starts, scale: float, causal: bool):
    """O [T, Hq, dv] and LSE [T, Hq] (NaN in rows that belong to no sequence); float64 caches [pages, Hkv, page, d].
    Keys in a page that is not there are not visible."""
    T, hq, _ = q.shape
    hkv, page, dv = k_cache.shape[1], k_cache.shape[2], v_cache.shape[3]
    o, lse = np.full((T, hq, dv), np.nan), np.full((T, hq), np.nan)
    for b in range(len(kv_lens)):
        q0, q1, n = int(q_starts[b]), int(q_starts[b + 1]), int(kv_lens[b])
        if q1 == q0:
            continue
        k, there = paged_rows(k_cache, table[b], n, page)
        v, _ = paged_rows(v_cache, table[b], n, page)
        for h in range(hq):
            g = h // (hq // hkv)
            if there.all():
                o[q0:q1, h], lse[q0:q1, h] = attention_head(q[q0:q1, h], k[:, g], v[:, g], scale, causal)
                continue
            for i in range(q1 - q0):  # rows one by one: each sees its own subset
                seen = there & ((np.arange(n) <= n - (q1 - q0) + i) | (not causal))
                r = attention_head(q[q0 + i:q0 + i + 1, h], k[seen, g], v[seen, g], scale, False)
                o[q0 + i, h], lse[q0 + i, h] = r[0][0], r[1][0]
    return o, lse
