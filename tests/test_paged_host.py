"""Paged cache on the host: every argument that is refused is refused before any HIP call (no GPU needed), the workspace
formula, and the oracle of the paged tests against closed forms."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import naive_attention
from oracle.paged import paged_attention, rotate, token_positions

P = 0x7F0000000000  # never dereferenced


def cache(**kw):
    a = dict(K=P, V=P + 0x10000, k_scale=None, v_scale=None, k_page=2 * 16 * 128, k_head=16 * 128, k_slot=128,
             v_page=2 * 16 * 128, v_head=16 * 128, v_slot=128, n_pages=8, page_size=16, Hkv=2, d_qk=128, d_v=128, type=0)
    a.update(kw)
    return fa.PagedCache(**a)


def batch(**kw):
    a = dict(block_table=P, table_stride=4, kv_lens=P, q_starts=P, B=3, max_blocks=4, T=5)
    a.update(kw)
    return fa.PagedBatch(**a)


def append(c=None, b=None, K=P, V=P, Q=P, Q_out=P, Hq=4, strides=(512, 128) * 2 + (256, 128) * 2, cos_sin=P, n_pos=64,
           begin=0, rot=128, inter=False):
    return fa.fa_kv_append(c or cache(), b or batch(), K, V, Q, Q_out, Hq, strides and fa.AppendStrides(*strides), cos_sin,
                           n_pos, begin, rot, inter, None)


def attend(c=None, b=None, Q=P, O=P, LSE=P, Hq=4, strides=(512, 128, 512, 128), max_q=2, path=0, scale=0.1, ws=P, nbytes=1 << 30):
    return fa.fa_fwd_paged(c or cache(), b or batch(), Q, O, LSE, Hq, strides and fa.PagedStrides(*strides), max_q, path, scale, True,
                           ws, nbytes, None)


SHAPE, UNSUPPORTED, NULL = fa.FA_ERR_BAD_SHAPE, fa.FA_ERR_UNSUPPORTED, fa.FA_ERR_NULL_POINTER
BOTH = [  # (cache changes, batch changes, status) of both entry points
    (dict(n_pages=-1), {}, SHAPE), (dict(Hkv=0), {}, SHAPE), (dict(Hkv=3), {}, SHAPE),
    ({}, dict(B=-1), SHAPE), ({}, dict(T=-1), SHAPE), ({}, dict(max_blocks=-1), SHAPE), ({}, dict(table_stride=-1), SHAPE),
    (dict(page_size=1 << 20), dict(max_blocks=1025), SHAPE), ({}, dict(T=2 ** 30), SHAPE),
    (dict(d_qk=96), {}, UNSUPPORTED), (dict(d_v=64), {}, UNSUPPORTED),
    (dict(page_size=0), {}, UNSUPPORTED), (dict(page_size=8), {}, UNSUPPORTED), (dict(page_size=48), {}, UNSUPPORTED),
    (dict(type=2), {}, UNSUPPORTED), (dict(k_scale=P), {}, UNSUPPORTED),
    (dict(K=None), {}, NULL), (dict(V=None), {}, NULL), ({}, dict(block_table=None), NULL), ({}, dict(kv_lens=None), NULL),
    ({}, dict(q_starts=None), NULL),
    (dict(K=P + 8), {}, UNSUPPORTED), (dict(k_slot=132), {}, UNSUPPORTED), (dict(v_page=4097), {}, UNSUPPORTED),
    ({}, dict(kv_lens=P + 2), UNSUPPORTED),
    (dict(k_slot=64), {}, SHAPE), (dict(v_page=-4096), {}, SHAPE), (dict(k_slot=1 << 27), {}, SHAPE),
    (dict(type=1, k_slot=136), {}, UNSUPPORTED), (dict(k_page=1 << 60), {}, SHAPE),
]


@pytest.mark.parametrize("ch,bt,status", BOTH, ids=str)
def test_both_refuse(ch, bt, status):
    page = ch.get("page_size", 16)
    n_pos = max(64, page * bt.get("max_blocks", 4))
    assert append(cache(**ch), batch(**bt), n_pos=min(n_pos, 2 ** 31 - 1), rot=64) == status
    assert attend(cache(**ch), batch(**bt)) == status


def test_append_refuses():
    assert append(strides=None) == NULL
    assert fa.fa_kv_append(None, batch(), P, P, P, P, 4, fa.AppendStrides(), P, 64, 0, 128, False, None) == NULL
    assert append(n_pos=63) == SHAPE           # a position could have no row
    assert append(n_pos=-1, rot=0) == SHAPE
    assert append(begin=16) == SHAPE           # past the head
    assert append(rot=-16) == SHAPE
    assert append(Hq=3) == SHAPE
    assert append(begin=4, rot=64) == UNSUPPORTED
    assert append(rot=24) == UNSUPPORTED and append(rot=4, inter=True) == UNSUPPORTED
    for kw in ("K", "V", "Q", "Q_out", "cos_sin"):
        assert append(**{kw: None}) == NULL, kw
        assert append(**{kw: P + 8}) == UNSUPPORTED, kw
    assert append(strides=(512, 128, 512, 128, 256, 127, 256, 128)) == UNSUPPORTED
    assert append(strides=(-512, 128, 512, 128, 256, 128, 256, 128)) == UNSUPPORTED
    # Places that coincide: pages, heads inside a page, a broadcast head.
    assert append(cache(k_page=4095 // 8 * 8)) == SHAPE
    assert append(cache(v_head=128)) == SHAPE and append(cache(k_head=0)) == SHAPE
    # Nothing to do: no HIP call.
    assert append(b=batch(T=0)) == fa.FA_OK and append(b=batch(B=0)) == fa.FA_OK


def test_attend_refuses():
    assert attend(strides=None) == NULL
    assert fa.fa_fwd_paged(cache(), None, P, P, P, 4, fa.PagedStrides(), 1, 0, 0.1, True, P, 1 << 30, None) == NULL
    assert attend(Hq=3) == SHAPE and attend(max_q=-1) == SHAPE
    assert attend(path=3) == UNSUPPORTED and attend(path=-1) == UNSUPPORTED
    assert attend(cache(Hkv=1), batch(T=2 ** 24, max_blocks=2 ** 20), Hq=64) == SHAPE  # more work than 32 bits count
    assert attend(Q=None) == NULL and attend(O=None) == NULL
    for scale in (float("nan"), float("inf"), 3e38):
        assert attend(scale=scale) == fa.FA_ERR_BAD_SCALE
    assert attend(Q=P + 4) == UNSUPPORTED and attend(O=P + 2) == UNSUPPORTED and attend(LSE=P + 2) == UNSUPPORTED
    assert attend(strides=(512, 128, 512, 100)) == UNSUPPORTED
    need = fa.fa_fwd_paged_workspace_bytes(3, 5, 256 * 16, 4, 2, 128, 128, 0, 2)
    long = batch(max_blocks=256, table_stride=256)
    assert attend(b=long, ws=None) == fa.FA_ERR_WORKSPACE and attend(b=long, nbytes=need - 1) == fa.FA_ERR_WORKSPACE
    assert attend(b=long, ws=P + 8, nbytes=need) == UNSUPPORTED
    assert attend(b=batch(T=0)) == fa.FA_OK and attend(b=batch(B=0)) == fa.FA_OK and attend(Hq=0) == fa.FA_OK


def test_workspace_bytes():
    def f(B, T, *a, keys=4096, path=0):
        return fa.fa_fwd_paged_workspace_bytes(B, T, keys, *a, path)

    assert f(1, 0, 4, 2, 128, 128, 0, 1) == 0 and f(0, 1, 4, 2, 128, 128, 0, 1) == 0 and f(1, 1, 3, 2, 128, 128, 0, 1) == 0
    assert f(1, 1, 4, 2, 96, 96, 0, 1) == 0 and f(1, 1, 4, 2, 64, 64, 7, 1) == 0 and f(1, 1, 4, 2, 64, 64, 0, -1) == 0
    one, most = f(1, 1, 4, 1, 128, 128, 0, 1), f(8, 8, 4, 1, 128, 128, 0, 1)
    assert 0 < one < most < 1 << 26 and 0 < f(10 ** 6, 10 ** 6, 4, 1, 128, 128, 0, 1) < 1 << 26
    assert f(1, 1, 4, 1, 128, 128, 0, 1, keys=-1) == 0
    # A chunk beside single tokens needs places for both kernels, unless the table holds too little for that for many
    # rows; enough equal prompts need none at all.
    assert f(8, 500, 4, 1, 128, 128, 0, 493, keys=65536) > f(8, 500, 4, 1, 128, 128, 0, 493, keys=1024)
    assert f(8, 80000, 32, 8, 128, 128, 0, 10000) == 0
    assert f(1, 1, 4, 1, 128, 128, 0, 1, path=3) == 0
    few, many = (f(8, 500, 4, 1, 128, 128, 0, 493, keys=65536, path=x) for x in (1, 2))
    assert 0 < few < many and few + many >= f(8, 500, 4, 1, 128, 128, 0, 493, keys=65536)


def test_structures_match_the_header():
    assert ctypes.sizeof(fa.PagedCache) == 4 * 8 + 6 * 8 + 6 * 4 and ctypes.sizeof(fa.PagedBatch) == 4 * 8 + 3 * 4 + 4


def test_tensors_that_are_refused():
    """The torch entry points: types, shapes, devices (a CPU tensor is refused)."""
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    c = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t, n, s = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.kv_append(k, k, c, c, t, n, s)
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.forward_paged(k, c, c, t, n, s)
    with pytest.raises(ValueError, match="4-d torch tensor"):
        fa.forward_paged(k, c.float(), c, t, n, s)
    with pytest.raises(ValueError, match="3-d bfloat16"):
        fa.forward_paged(k[0], c, c, t, n, s)
    with pytest.raises(ValueError, match="3-d bfloat16"):
        fa.kv_append(None, k, c, c, t, n, s)


# ---- the oracle -------------------------------------------------------------------------------------

def test_oracle_rotation():
    rng = np.random.RandomState(0)
    x, a = rng.randn(5, 12), rng.rand(3) * 6
    for inter in (False, True):
        y = rotate(x, np.cos(a), np.sin(a), 4, inter)
        assert np.array_equal(y[:, :4], x[:, :4]) and np.array_equal(y[:, 10:], x[:, 10:])
        assert np.allclose((y ** 2).sum(1), (x ** 2).sum(1), atol=1e-12)       # a turn keeps lengths
        assert np.allclose(rotate(y, np.cos(a), -np.sin(a), 4, inter), x, atol=1e-12)
        i, j = (4, 5) if inter else (4, 7)
        z = (x[:, i] + 1j * x[:, j]) * np.exp(1j * a[0])
        assert np.allclose(y[:, i], z.real) and np.allclose(y[:, j], z.imag)


def test_oracle_positions():
    assert token_positions([0, 2, 2, 5], [7, 3, 2]) == [(0, 5), (0, 6), (-1, -1), (2, 0), (2, 1)]


@pytest.mark.parametrize("causal", [True, False])
def test_oracle_paged_attention_is_attention_over_the_gathered_keys(causal):
    rng = np.random.RandomState(1)
    kc, vc = rng.randn(9, 2, 4, 6), rng.randn(9, 2, 4, 3)
    table, lens, starts = np.array([[5, 1, 8], [0, 7, 2]]), [10, 7], [0, 3, 4]
    q = rng.randn(4, 4, 6)
    o, lse = paged_attention(q, kc, vc, table, lens, starts, 0.3, causal)
    for b in range(2):
        flat = lambda c: np.concatenate([c[p] for p in table[b]], axis=1)[None, :, : lens[b]]  # noqa: E731
        q_b = q[starts[b]:starts[b + 1]].transpose(1, 0, 2)[None]
        ro, rl = naive_attention(q_b, flat(kc), flat(vc), 0.3, causal)
        assert np.allclose(o[starts[b]:starts[b + 1]], ro[0].transpose(1, 0, 2), atol=1e-13)
        assert np.allclose(lse[starts[b]:starts[b + 1]], rl[0].T, atol=1e-13)
    # A page that is not there: the same as the sequence without its keys (not causal).
    table2 = np.array([[5, -1, 8], [0, 7, 2]])
    o2, _ = paged_attention(q, kc, vc, table2, lens, starts, 0.3, False)
    keep = [0, 1, 2, 3, 8, 9]
    k0, v0 = (np.concatenate([c[p] for p in table[0]], axis=1)[None, :, keep] for c in (kc, vc))
    ro, _ = naive_attention(q[:3].transpose(1, 0, 2)[None], k0, v0, 0.3, False)
    assert np.allclose(o2[:3], ro[0].transpose(1, 0, 2), atol=1e-13)
