"""Around the paged cache in float64 and whole numbers: rotations by positions of several axes, masks of drafted trees,
tokens closed up and pages copied, and attention with every way of changing or hiding scores.

TEST INFRASTRUCTURE ONLY (see the package docstring). Everything is written token by token from the definitions.
"""

from __future__ import annotations

import numpy as np

from .paged import paged_rows, rotate


def rows_of(position, pair_axes, n_pairs: int, n_pos: int):
    """The table row of each pair of a token that stands at `position` [axes]."""
    axes = [0] * n_pairs if pair_axes is None else [min(int(a), len(position) - 1) for a in pair_axes]
    return [min(max(int(position[a]), 0), n_pos - 1) for a in axes]


def rotate_at(x, table, rows, begin: int, interleaved: bool, sign: float = 1.0):
    """x [H, d] turned: pair c by the angle of row rows[c], column c, of the table [n_pos, rot]."""
    half = table.shape[1] // 2
    cos = [table[r, c] for c, r in enumerate(rows)]
    sin = [sign * table[r, half + c] for c, r in enumerate(rows)]
    return rotate(x, np.array(cos), np.array(sin), begin, interleaved)


def paths(parents):
    """Of every token of one tree: the set of itself and its ancestors."""
    out = []
    for i, p in enumerate(parents):
        out.append({i} | (out[p] if 0 <= p < i else set()))
    return out


def compact(cache, table, kv_lens, q_starts, kept, n_kept):
    """The cache [pages, H, page, d] after the kept tokens closed up, and the new lengths."""
    out, page = cache.copy(), cache.shape[2]
    lens = []
    for b, kv in enumerate(kv_lens):
        n = max(0, q_starts[b + 1] - q_starts[b])
        base, m = kv - n, min(max(n_kept[b], 0), len(kept[b]), n)
        for i in range(m):
            k = int(kept[b][i])
            a, z = base + k, base + i
            if not 0 <= k < n or a < 0 or z < 0:
                continue
            pa, pz = table[b][a // page], table[b][z // page]
            if 0 <= pa < len(cache) and 0 <= pz < len(cache):
                out[pz, :, z % page] = cache[pa, :, a % page]
        lens.append(max(base + m, 0))
    return out, lens


def visible(n: int, kv: int, causal=True, window=None, prefix=0, tree=None):
    """Which of kv keys each of the last n tokens sees, [n, kv]. tree [n, n]: which new tokens each sees."""
    out = np.zeros((n, kv), dtype=bool)
    for i in range(n):
        p = kv - n + i
        for j in range(kv):
            if tree is not None:
                out[i, j] = j < kv - n or (j - (kv - n) < tree.shape[1] and tree[i, j - (kv - n)])
            else:
                inside = (j <= p or not causal) and (window is None or abs(p - j) < window)
                out[i, j] = j < prefix or inside
    return out


def paged_attention(q, k_cache, v_cache, table, kv_lens, q_starts, scale, causal=True, cap=None, slopes=None, window=None,
                    prefix=None, tree=None):
    """O [T, Hq, dv], LSE [T, Hq] (NaN in rows of no sequence), and of every row the mass sum_j p_j |v_j| [T, Hq, dv];
    tree: [T, any] booleans. Scores x = scale q.k, then cap tanh(x / cap), then x - slope |p - j|."""
    T, hq, _ = q.shape
    hkv, page, dv = k_cache.shape[1], k_cache.shape[2], v_cache.shape[3]
    o, lse, mass = np.full((T, hq, dv), np.nan), np.full((T, hq), np.nan), np.full((T, hq, dv), np.nan)
    for b in range(len(kv_lens)):
        q0, q1, kv = int(q_starts[b]), int(q_starts[b + 1]), int(kv_lens[b])
        n = q1 - q0
        if n <= 0:
            continue
        k, there = paged_rows(k_cache, table[b], kv, page)
        v, _ = paged_rows(v_cache, table[b], kv, page)
        k, v = np.where(there[:, None, None], k, 0.0), np.where(there[:, None, None], v, 0.0)
        seen = visible(n, kv, causal, window, int(prefix[b]) if prefix is not None else 0,
                       tree[q0:q1] if tree is not None else None) & there
        far = np.abs(kv - n + np.arange(n)[:, None] - np.arange(kv))
        for h in range(hq):
            g = h // (hq // hkv)
            x = scale * (q[q0:q1, h] @ np.where(seen.any(0)[:, None], k[:, g], 0.0).T)
            if cap is not None:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - float(slopes[h]) * far
            x = np.where(seen, x, -np.inf)
            top = x.max(axis=1, keepdims=True, initial=-np.inf)
            e = np.exp(x - np.where(np.isneginf(top), 0.0, top))
            total = e.sum(axis=1, keepdims=True)
            some = total > 0
            p = np.where(some, e / np.where(some, total, 1.0), 0.0)
            vg = np.where(seen.any(0)[:, None], v[:, g], 0.0)
            o[q0:q1, h], mass[q0:q1, h] = p @ vg, p @ np.abs(vg)
            with np.errstate(divide="ignore"):
                lse[q0:q1, h] = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)[:, 0]
    return o, lse, mass
