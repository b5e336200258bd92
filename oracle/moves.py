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
    """Which of kv keys each of the last n tokens sees, [n, kv]. tree [n, any]: which new tokens each sees."""
    p, j = kv - n + np.arange(n)[:, None], np.arange(kv)[None]
    if tree is None:
        inside = (j <= p) if causal else np.ones((n, kv), dtype=bool)
        if window is not None:
            inside = inside & (np.abs(p - j) < window)
        return inside | (j < prefix)
    out = np.broadcast_to(j < kv - n, (n, kv)).copy()
    for i in range(min(n, tree.shape[1])):
        if kv - n + i >= 0:
            out[:, kv - n + i] = tree[:, i]
    return out


def tree_bits(mask):
    """Words [T, W] as booleans [T, 32 W]."""
    return (np.asarray(mask).astype(np.int64)[:, :, None] >> np.arange(32) & 1).astype(bool).reshape(len(mask), -1)


class Attention:
    """o [T, Hq, dv] and lse [T, Hq] (NaN in rows of no sequence), and for the bars of a test, per row of every head: mass =
    sum_j p_j |v_j|, off_v = sum_j p_j e_j |v_j|, off = sum_j p_j e_j, with p the probabilities and e_j = 2^-24 d scale sum_i |q_i k_ji| +
    2^-21 (1 + |x_j| + |bias_j| + cap): how far fp32 arithmetic may move the score of key j; and keys [T]: how many the row has."""

    def __init__(self, T, hq, dv):
        self.o, self.lse = np.full((T, hq, dv), np.nan), np.full((T, hq), np.nan)
        self.mass, self.off_v = np.zeros((T, hq, dv)), np.zeros((T, hq, dv))
        self.off, self.vmax, self.keys = np.zeros((T, hq)), np.zeros((T, hq)), np.zeros(T)


def paged_attention(q, k_cache, v_cache, table, kv_lens, q_starts, scale, causal=True, cap=None, slopes=None, window=None,
                    prefix=None, tree=None):
    """The attention of fa_fwd_paged_ex in float64, as an :class:`Attention`; tree: booleans [T, any]. Scores x = scale q.k, then
    cap tanh(x / cap), then x - slope |p - j|."""
    T, hq, d = q.shape
    hkv, page, dv = k_cache.shape[1], k_cache.shape[2], v_cache.shape[3]
    r = Attention(T, hq, dv)
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
        used = seen.any(0)[:, None]
        far = np.abs(kv - n + np.arange(n)[:, None] - np.arange(kv))
        for h in range(hq):
            g = h // (hq // hkv)
            kg, vg = np.where(used, k[:, g], 0.0), np.where(used, v[:, g], 0.0)
            x = scale * (q[q0:q1, h] @ kg.T)
            e = 2.0 ** -24 * d * abs(scale) * (np.abs(q[q0:q1, h]) @ np.abs(kg).T) + 2.0 ** -21 * (1 + np.abs(x) + (cap or 0.0))
            if cap is not None:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - float(slopes[h]) * far
                e = e + 2.0 ** -21 * abs(float(slopes[h])) * far
            x = np.where(seen, x, -np.inf)
            top = x.max(axis=1, keepdims=True, initial=-np.inf)
            w = np.exp(x - np.where(np.isneginf(top), 0.0, top))
            total = w.sum(axis=1, keepdims=True)
            some = total > 0
            total = np.where(some, total, 1.0)
            p = np.where(some, w / total, 0.0)
            r.o[q0:q1, h], r.mass[q0:q1, h] = p @ vg, p @ np.abs(vg)
            r.off_v[q0:q1, h], r.off[q0:q1, h] = (p * e) @ np.abs(vg), (p * e).sum(1)
            r.vmax[q0:q1, h] = np.abs(vg).max(initial=0.0)
            r.lse[q0:q1, h] = np.where(some, top + np.log(total), -np.inf)[:, 0]
        r.keys[q0:q1] = seen.sum(1)
    return r
