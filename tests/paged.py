"""Helpers of the paged-cache tests: a batch over a cache with pages in no order, and tolerances.

Tolerances. bf16 has a half step of 2^-8 relative to the value, fp16 2^-11, e4m3 2^-4 (2^-10 absolute below its
smallest normal value), fp32 2^-24.
* O: P enters the P V product rounded to bf16 (fp16 over an e4m3 cache), which moves O by at most 2^-8 max|V| over the
  visible keys (2^-11), and O is rounded once, 2^-8 |O| <= 2^-8 max|V|; fp32 sums and exponentials 1e-5 max|V|.
* LSE: a score is an fp32 sum of d products, off by at most d 2^-24 sum|q_i k_i| scale <= d^2 2^-24 max|q| max|k| scale; the
  sums, logarithm and one multiplication by scale * log2(e) add 2^-20 (1 + |LSE| + max|score|).
* An appended element: fp32 products and sums of a pair (2^-22 (|x| + |y|)) and one rounding.
"""

from __future__ import annotations

import numpy as np
import torch

import paper_2609_21264_amd as fa
from oracle.paged import paged_attention, paged_rows

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Batch:
    """A packed batch: ``new`` and ``keys`` per sequence, over a cache whose unused slots hold NaN."""

    def __init__(self, new, keys, Hq, Hkv, dqk, dv, page=16, fp8=False, seed=0, device="cuda:0", spare=3, extra=0,
                 order="hnd", sigma=1.0, blocks=None):
        g = torch.Generator().manual_seed(seed)
        self.new, self.keys, self.page, self.fp8, self.device = list(new), list(keys), page, fp8, device
        self.Hq, self.Hkv, self.dqk, self.dv = Hq, Hkv, dqk, dv
        self.T = sum(new) + extra  # `extra` tokens behind the last sequence
        need = [-(-k // page) for k in keys]
        self.n_pages = sum(need) + spare
        blocks = blocks or max(need + [1])
        perm = torch.randperm(self.n_pages, generator=g, dtype=torch.int32)
        self.table = torch.full((len(keys), blocks), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.q_starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
        self.kv_lens = torch.tensor(keys, dtype=torch.int32)

        def randn(*shape):
            return torch.randn(*shape, generator=g) * sigma

        self.q = randn(self.T, Hq, dqk).to(BF16)
        self.k, self.v = randn(self.T, Hkv, dqk).to(BF16), randn(self.T, Hkv, dv).to(BF16)
        self.k_scale = self.v_scale = None
        kc, vc = randn(self.n_pages, Hkv, page, dqk), randn(self.n_pages, Hkv, page, dv)
        if fp8:
            self.k_scale, self.v_scale = 0.01 + 0.01 * torch.rand(Hkv, generator=g), 0.01 + 0.01 * torch.rand(Hkv, generator=g)
            kc, vc = kc / self.k_scale[:, None, None], vc / self.v_scale[:, None, None]
            kc, vc = kc.clamp(-448, 448).to(E4M3), vc.clamp(-448, 448).to(E4M3)
        else:
            kc, vc = kc.to(BF16), vc.to(BF16)
        used = torch.zeros(self.n_pages, page, dtype=torch.bool)
        for b, k in enumerate(keys):
            pos = torch.arange(k)
            used[self.table[b, pos // page].long(), pos % page] = True
        raw = torch.uint8 if fp8 else torch.int16
        nan = 0x7F if fp8 else 0x7FC0
        for c in (kc, vc):  # slots that hold no key
            c.view(raw).permute(0, 2, 1, 3)[~used] = nan
        self.k_cache, self.v_cache = kc, vc
        self.used = used
        self._to(device, order)

    def _to(self, device, order):
        for name in ("q", "k", "v", "table", "kv_lens", "q_starts", "k_cache", "v_cache", "k_scale", "v_scale"):
            t = getattr(self, name)
            setattr(self, "d_" + name, None if t is None else t.to(device))
        if order == "nhd":  # slots of a page outside its heads
            for name in ("d_k_cache", "d_v_cache"):
                raw = getattr(self, name)
                raw = raw.view(torch.uint8) if self.fp8 else raw
                t = raw.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
                setattr(self, name, t.view(E4M3) if self.fp8 else t)

    def values(self, cache, scale):
        x = f64(cache)
        return x * f64(scale)[:, None, None] if scale is not None else x

    def attend(self, **kw):
        kw.setdefault("max_q", max(self.new + [0]))
        return fa.forward_paged(self.d_q, self.d_k_cache, self.d_v_cache, self.d_table, self.d_kv_lens, self.d_q_starts,
                                k_scale=self.d_k_scale, v_scale=self.d_v_scale, **kw)

    def append(self, **kw):
        return fa.kv_append(self.d_k, self.d_v, self.d_k_cache, self.d_v_cache, self.d_table, self.d_kv_lens,
                            self.d_q_starts, k_scale=self.d_k_scale, v_scale=self.d_v_scale, **kw)

    def oracle(self, scale, causal):
        return paged_attention(f64(self.q), self.values(self.k_cache, self.k_scale),
                               self.values(self.v_cache, self.v_scale), self.table.numpy(), self.kv_lens.numpy(),
                               self.q_starts.numpy(), scale, causal)

    def check(self, o, lse, scale, causal, what=""):
        """O and LSE against the oracle, within the bars of the module's docstring."""
        torch.cuda.synchronize()
        o_ref, lse_ref = self.oracle(scale, causal)
        n = int(self.q_starts[-1])
        o, lse, o_ref, lse_ref = f64(o)[:n], f64(lse)[:n], o_ref[:n], lse_ref[:n]
        first = int(self.q_starts[0])
        o, lse, o_ref, lse_ref = o[first:], lse[first:], o_ref[first:], lse_ref[first:]
        group = self.Hq // self.Hkv
        kc, vc = self.values(self.k_cache, self.k_scale), self.values(self.v_cache, self.v_scale)
        q64 = f64(self.q)
        bar_o, bar_l = np.zeros(lse.shape), np.zeros(lse.shape)
        for b, (q0, q1) in enumerate(zip(self.q_starts[:-1].tolist(), self.q_starts[1:].tolist())):
            if q1 == q0:
                continue
            k, there = paged_rows(kc, self.table[b].numpy(), int(self.kv_lens[b]), self.page)
            v, _ = paged_rows(vc, self.table[b].numpy(), int(self.kv_lens[b]), self.page)
            k, v = k[there], v[there]
            kmax = np.abs(k).max(axis=(0, 2)) if len(k) else np.zeros(self.Hkv)
            vmax = np.abs(v).max(axis=(0, 2)) if len(v) else np.zeros(self.Hkv)
            qmax = np.abs(q64[q0:q1]).max(axis=2)
            top = self.dqk * np.repeat(kmax, group) * qmax * abs(scale)  # no score is larger
            bar_o[q0 - first:q1 - first] = ((2.0 ** -11 if self.fp8 else 2.0 ** -8) + 2.0 ** -8 + 1e-5) * np.repeat(vmax, group)
            bar_l[q0 - first:q1 - first] = self.dqk * 2.0 ** -24 * top + 2.0 ** -20 * (1 + top)
        empty = np.isneginf(lse_ref)
        assert np.array_equal(np.isneginf(lse), empty), f"{what}: rows without a visible key differ"
        assert np.isfinite(o).all() and np.isfinite(lse[~empty]).all(), f"{what}: not finite"
        assert np.all(o[empty] == 0), f"{what}: O of a row without a visible key"
        off = np.abs(o - o_ref) - bar_o[..., None]
        assert off.max(initial=-1) <= 0, f"{what}: O off by {np.abs(o - o_ref).max():.3e}, bar {bar_o.max():.3e}"
        # fp32 scores feed exp: what an LSE bar allows moves O by no more than that bar times max|V|, far inside bar_o.
        loff = np.abs(lse[~empty] - lse_ref[~empty]) - (bar_l + 2.0 ** -20 * np.abs(np.where(empty, 0, lse_ref)))[~empty]
        assert loff.max(initial=-1) <= 0, f"{what}: LSE off by {np.abs(lse[~empty] - lse_ref[~empty]).max():.3e}"


def cos_sin_table(positions, rot, seed=0):
    """An fp32 table of arbitrary angles (any table is allowed)."""
    a = torch.rand(positions, rot // 2, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 6.3
    return torch.cat([a.cos(), a.sin()], dim=1).float()
