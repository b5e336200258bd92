"""Tests of the paged attention by probability mass.

V is one-hot: dim c of a key's value is 1 where the key belongs to class c, so O[..., c] is the class's share of the row's
probability. Sums of i.i.d. values shrink as keys are added while a bar relative to max|V| does not; here every term is
positive, so the roundings bound the relative error of each output element:
* P is rounded once before it meets V, by 2^-8 of it (bf16) or 2^-11 of it, at least 2^-32 of the row's largest (fp16 over
  an e4m3 cache; absolute, for each key); all terms of a class have its sign, so its sum moves by no more.
* O is rounded once: 2^-8 of it.
* A score is an fp32 sum of d products, off by at most d 2^-24 S for S = the largest sum |q_i k_i| scale of the row's keys, and
  the exponentials, sums and joins add 2^-20 (1 + S); both enter P and the row sum.
Classes: "blocks", runs of keys of odd length, so that a tile, half or part that is lost, doubled, misplaced or weighted wrongly
shows in its own dims; "residues", the key's position modulo d_v, so that keys mixed up inside a tile show.
"""

from __future__ import annotations

import numpy as np
import torch

from oracle.paged import paged_rows
from paged import Batch, f64

KINDS = ["blocks", "residues"]


def classes(kind, n, dv):
    """The class of keys 0 .. n-1; blocks of an odd length."""
    pos = np.arange(n)
    if kind == "residues":
        return pos % dv
    return pos // (-(-max(n, 1) // dv) | 1)


def mass_batch(kind, new, keys, Hq, Hkv, dqk, dv, page=16, fp8=False, **kw):
    bt = Batch(new, keys, Hq, Hkv, dqk, dv, page, fp8, **kw)
    raw = bt.v_cache.view(torch.uint8 if fp8 else torch.int16)
    one = torch.tensor(0x38 if fp8 else 0x3F80, dtype=raw.dtype)
    for b, n in enumerate(keys):
        pos = torch.arange(n)
        rows = torch.zeros(n, dv, dtype=raw.dtype)
        rows[pos, torch.from_numpy(classes(kind, n, dv))] = one
        raw[bt.table[b, pos // page].long(), :, pos % page] = rows[:, None].expand(n, Hkv, dv)
    bt.kind = kind
    bt._to(bt.device, kw.get("order", "hnd"))
    return bt


def reference(bt, scale, causal, drop=None):
    """O in float64 and the bar of each element; `drop` (a CPU test's mistake): keys [a, b) of every sequence are lost."""
    group = bt.Hq // bt.Hkv
    kc = bt.values(bt.k_cache, bt.k_scale)
    q = f64(bt.q)
    vs = f64(bt.v_scale) if bt.v_scale is not None else np.ones(bt.Hkv)
    o, bar = np.zeros((bt.T, bt.Hq, bt.dv)), np.zeros((bt.T, bt.Hq, bt.dv))
    for b, n in enumerate(bt.keys):
        q0, q1 = int(bt.q_starts[b]), int(bt.q_starts[b + 1])
        if q1 == q0 or n == 0:
            continue
        k, there = paged_rows(kc, bt.table[b].numpy(), n, bt.page)
        if drop is not None:
            there = there & ((np.arange(n) < drop[0]) | (np.arange(n) >= drop[1]))
        hot = np.zeros((n, bt.dv))
        hot[np.arange(n), classes(bt.kind, n, bt.dv)] = 1.0
        last = n - (q1 - q0) + np.arange(q1 - q0) if causal else np.full(q1 - q0, n - 1)
        seen = (np.arange(n)[None] <= last[:, None]) & there[None]
        for h in range(bt.Hq):
            g = h // group
            x = np.where(seen, q[q0:q1, h] @ k[:, g].T * scale, -np.inf)
            top = x.max(axis=1, keepdims=True)
            w = np.where(seen, np.exp(x - np.where(np.isneginf(top), 0.0, top)), 0.0)
            total = w.sum(axis=1, keepdims=True)
            w = w / np.where(total > 0, total, 1.0)
            big = (np.where(seen, np.abs(q[q0:q1, h]) @ np.abs(k[:, g]).T, 0.0) * abs(scale)).max(axis=1, keepdims=True)
            y = w @ hot * vs[g]
            rel = (2.0 ** -11 if bt.fp8 else 2.0 ** -8) + 2.0 ** -8 + 2 * (bt.dqk * 2.0 ** -24 * big + 2.0 ** -20 * (1 + big))
            o[q0:q1, h], bar[q0:q1, h] = y, rel * y + ((seen * 2.0 ** -32) @ hot * vs[g] if bt.fp8 else 0.0)
    return o, bar


def check_mass(bt, o, scale, causal, what=""):
    want, bar = reference(bt, scale, causal)
    first, last = int(bt.q_starts[0]), int(bt.q_starts[-1])
    o, want, bar = (f64(o) if isinstance(o, torch.Tensor) else o)[first:last], want[first:last], bar[first:last]
    off = np.abs(o - want) - bar
    assert off.max(initial=-1.0) <= 0, (f"{what}: mass off by {np.abs(o - want).max():.3e} at (token, head, class) "
                                        f"{np.unravel_index(np.argmax(off), off.shape)}")
