"""Positions of several axes, drafted trees and moves in the paged cache on the host: what is refused is refused before any
HIP call, and the oracle against closed forms."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import moves
from test_paged_host import NULL, P, SHAPE, UNSUPPORTED, batch, cache


def at(**kw):
    a = dict(positions=P, pair_axes=P, batch=0, token=3, axis=1, n_axes=3)
    a.update(kw)
    return fa.Positions(**a)


def append_at(c=None, b=None, pos="", K=P, V=P, Q=P, Q_out=P, Hq=4, strides=(512, 128) * 2 + (256, 128) * 2, cos_sin=P,
              n_pos=5, begin=0, rot=128, inter=False):
    return fa.fa_kv_append_at(c or cache(), b or batch(), K, V, Q, Q_out, Hq, fa.AppendStrides(*strides),
                              at() if pos == "" else pos, cos_sin, n_pos, begin, rot, inter, None)


def rotate(pos="", X=P, Y=P + 4096, B=2, H=3, S=5, d=64, strides=(960, 320, 64) * 2, cos_sin=P, n_pos=5, begin=0, rot=64,
           inter=False):
    return fa.fa_rotate(X, Y, B, H, S, d, strides and fa.RotateStrides(*strides), at() if pos == "" else pos, cos_sin, n_pos, begin,
                        rot, inter, False, None)


def test_append_at_refuses():
    assert append_at(pos=None) == NULL
    assert append_at(pos=at(n_axes=0)) == SHAPE and append_at(n_pos=0) == SHAPE and append_at(n_pos=-1, rot=0) == SHAPE
    for name in ("batch", "token", "axis"):
        assert append_at(pos=at(**{name: -1})) == SHAPE and append_at(pos=at(**{name: (1 << 40) + 1})) == SHAPE
    assert append_at(pos=at(positions=None)) == NULL and append_at(cos_sin=None) == NULL
    assert append_at(pos=at(positions=P + 2)) == UNSUPPORTED and append_at(pos=at(pair_axes=P + 1)) == UNSUPPORTED
    assert append_at(begin=16) == SHAPE and append_at(rot=24) == UNSUPPORTED and append_at(Hq=3) == SHAPE
    assert append_at(cache(page_size=8)) == UNSUPPORTED and append_at(cache(v_head=128)) == SHAPE
    assert append_at(b=batch(T=0)) == fa.FA_OK and append_at(b=batch(B=0)) == fa.FA_OK


def test_rotate_refuses():
    assert rotate(strides=None) == NULL
    for kw in (dict(B=-1), dict(H=-1), dict(S=-1), dict(d=-8), dict(B=1 << 20, H=1 << 6, S=1 << 6), dict(begin=8), dict(rot=-16),
               dict(pos=at(n_axes=0)), dict(n_pos=0), dict(pos=None, n_pos=4), dict(pos=at(positions=None), n_pos=4)):
        assert rotate(**kw) == SHAPE, kw
    for kw in (dict(d=68), dict(d=1032), dict(begin=4, rot=32), dict(rot=24), dict(rot=4, inter=True), dict(X=P + 8), dict(Y=P + 2),
               dict(cos_sin=P + 4), dict(strides=(960, 320, 63) * 2), dict(strides=(960, -320, 64) * 2),
               dict(pos=at(positions=P + 1)), dict(pos=at(pair_axes=P + 2))):
        assert rotate(**kw) == UNSUPPORTED, kw
    for kw in (dict(X=None), dict(Y=None), dict(cos_sin=None)):
        assert rotate(**kw) == NULL, kw
    for kw in (dict(B=0), dict(H=0), dict(S=0), dict(d=0, rot=0)):
        assert rotate(**kw) == fa.FA_OK, kw
    assert rotate(Y=P, rot=0) == fa.FA_OK  # in place and nothing turns


def tree(parents=P, starts=P, lens=P, B=3, T=9, max_keys=64, mask=P, words=1, stride=1, positions=P):
    return fa.fa_tree_mask(parents, starts, lens, B, T, max_keys, mask, words, stride, positions, None)


def test_tree_mask_refuses():
    for kw in (dict(B=-1), dict(T=-1), dict(B=2 ** 31 - 1), dict(max_keys=-1), dict(max_keys=(1 << 30) + 1), dict(words=0),
               dict(words=fa.FA_TREE_WORDS + 1, stride=100), dict(words=3, stride=2), dict(stride=(1 << 40) + 1)):
        assert tree(**kw) == SHAPE, kw
    for name in ("parents", "starts", "lens", "mask", "positions"):
        assert tree(**{name: None}) == NULL and tree(**{name: P + 2}) == UNSUPPORTED, name
    assert tree(B=0) == fa.FA_OK and tree(T=0) == fa.FA_OK


def compact(c=None, b=None, kept=P, stride=4, most=4, n_kept=P, out=P):
    return fa.fa_kv_compact(c or cache(), b or batch(), kept, stride, most, n_kept, out, None)


def copy(c=None, src=P, dst=P, n=3):
    return fa.fa_kv_copy(c or cache(), src, dst, n, None)


def test_moves_refuse():
    assert fa.fa_kv_compact(None, batch(), P, 4, 4, P, P, None) == NULL and fa.fa_kv_compact(cache(), None, P, 4, 4, P, P, None) == NULL
    assert compact(most=-1) == SHAPE and compact(stride=-1) == SHAPE and compact(b=batch(B=-1)) == SHAPE
    assert compact(cache(Hkv=1 << 25)) == SHAPE
    assert fa.fa_kv_copy(None, P, P, 3, None) == NULL and copy(n=-1) == SHAPE
    for ch, status in ((dict(n_pages=-1), SHAPE), (dict(Hkv=-1), SHAPE), (dict(d_qk=96), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED),
                       (dict(type=5), UNSUPPORTED), (dict(K=None), NULL), (dict(V=None), NULL), (dict(K=P + 8), UNSUPPORTED),
                       (dict(v_slot=132), UNSUPPORTED), (dict(k_page=4088), SHAPE), (dict(k_head=0), SHAPE)):
        assert compact(cache(**ch)) == status and copy(cache(**ch)) == status, ch
    for name in ("kept", "n_kept", "out"):
        assert compact(**{name: None}) == NULL and compact(**{name: P + 2}) == UNSUPPORTED, name
    for name in ("src", "dst"):
        assert copy(**{name: None}) == NULL and copy(**{name: P + 2}) == UNSUPPORTED, name
    assert compact(b=batch(B=0)) == fa.FA_OK and copy(n=0) == fa.FA_OK and copy(cache(n_pages=0)) == fa.FA_OK
    # More workgroups than one dimension of a grid holds; a page of more 16-byte chunks than 31 bits count.
    big = cache(page_size=1 << 14, Hkv=64, k_head=1 << 21, v_head=1 << 21, k_page=1 << 27, v_page=1 << 27)
    assert copy(big, n=1 << 12) == SHAPE
    huge = cache(page_size=1 << 20, Hkv=128, k_head=1 << 27, v_head=1 << 27, k_page=1 << 34, v_page=1 << 34)
    assert copy(huge, n=1) == SHAPE


def test_tensors_that_are_refused():
    z = dict(dtype=torch.int32)
    k, c = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t, n, s = torch.zeros(1, 2, **z), torch.zeros(1, **z), torch.zeros(2, **z)
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.rotate(k, torch.zeros(4, 64))
    with pytest.raises(ValueError, match="bfloat16"):
        fa.rotate(k.float(), torch.zeros(4, 64))
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.tree_mask(n, s, n)
    with pytest.raises(ValueError, match="1-d int32"):
        fa.tree_mask(n.float(), s, n)
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.kv_compact(c, c, t, n, s, t, n)
    with pytest.raises(ValueError, match="must be on a GPU"):
        fa.kv_copy(c, c, n, n)
    with pytest.raises(ValueError, match="1-d int32"):
        fa.kv_copy(c, c, n.long(), n)
    assert ctypes.sizeof(fa.Positions) == 2 * 8 + 3 * 8 + 8


# ---- the oracle -------------------------------------------------------------------------------------

def test_oracle_rows_and_rotation():
    assert moves.rows_of([4, -2, 99], [0, 1, 2, 7], 4, 50) == [4, 0, 49, 49] and moves.rows_of([3], None, 2, 9) == [3, 3]
    rng = np.random.RandomState(0)
    x, a = rng.randn(2, 8), rng.rand(5, 3) * 6
    table = np.concatenate([np.cos(a), np.sin(a)], axis=1)
    y = moves.rotate_at(x, table, [4, 0, 2], 2, False)
    z = (x[:, 3] + 1j * x[:, 6]) * np.exp(1j * a[0, 1])
    assert np.allclose(y[:, 3], z.real) and np.allclose(y[:, 6], z.imag)
    assert np.allclose(moves.rotate_at(y, table, [4, 0, 2], 2, False, -1.0), x, atol=1e-12)


def test_oracle_paths():
    assert moves.paths([-1, 0, 0, 2, 9, 5]) == [{0}, {0, 1}, {0, 2}, {0, 2, 3}, {4}, {5}]


def test_oracle_compact():
    c = np.arange(3 * 1 * 4 * 1).reshape(3, 1, 4, 1)
    out, lens = moves.compact(c, [[2, 0]], [7], [0, 4], [[1, 3]], [2])  # keys 0-2 cached, new ones 3-6; 4 and 6 close up
    assert out[2, 0, 3, 0] == c[0, 0, 0, 0] and out[0, 0, 0, 0] == c[0, 0, 2, 0] and lens == [5]
    assert (out != c).sum() == 2


def test_oracle_visible():
    causal = moves.visible(2, 5)
    assert causal.tolist() == [[True] * 4 + [False], [True] * 5]
    assert moves.visible(2, 5, window=2).tolist() == [[False, False, True, True, False], [False, False, False, True, True]]
    assert moves.visible(1, 5, window=1, prefix=2).tolist() == [[True, True, False, False, True]]
    assert moves.visible(2, 5, causal=False, window=2).tolist() == [[False, False, True, True, True], [False] * 3 + [True] * 2]
    assert moves.visible(3, 3, prefix=2).tolist() == [[True, True, False], [True, True, False], [True] * 3]
    tree = np.array([[True, False], [False, True]])
    assert moves.visible(2, 4, tree=tree).tolist() == [[True, True, True, False], [True, True, False, True]]


def test_oracle_attention():
    """Against naive attention where nothing is set, and by hand for a cap, a bias and a tree."""
    from oracle.paged import paged_attention as plain

    rng = np.random.RandomState(1)
    kc, vc = rng.randn(9, 2, 4, 6), rng.randn(9, 2, 4, 3)
    table, lens, starts, q = np.array([[5, 1, 8], [0, 7, 2]]), [10, 7], [0, 3, 4], rng.randn(4, 4, 6)
    for causal in (True, False):
        o, lse = plain(q, kc, vc, table, lens, starts, 0.3, causal)
        r = moves.paged_attention(q, kc, vc, table, lens, starts, 0.3, causal)
        assert np.allclose(r.o, o, atol=1e-13) and np.allclose(r.lse, lse, atol=1e-13)
    bits = moves.tree_bits(np.array([[1], [3], [5], [-2 ** 31]], dtype=np.int32))
    assert bits.shape == (4, 32) and bits[:3, :3].tolist() == [[True, False, False], [True, True, False], [True, False, True]]
    assert bits[3].tolist() == [False] * 31 + [True]
    r = moves.paged_attention(q, kc, vc, table, lens, starts, 0.3, cap=0.8, tree=bits)
    keys = np.concatenate([kc[p] for p in table[0]], axis=1)[:, [0, 1, 2, 3, 4, 5, 6, 7, 9]]  # token 2 sees 0 and 2
    vals = np.concatenate([vc[p] for p in table[0]], axis=1)[:, [0, 1, 2, 3, 4, 5, 6, 7, 9]]
    w = np.exp(0.8 * np.tanh(0.3 * keys[1] @ q[2, 3] / 0.8))
    assert np.allclose(r.o[2, 3], (w / w.sum()) @ vals[1]) and np.allclose(r.lse[2, 3], np.log(w.sum()))
    assert r.keys.tolist() == [8, 9, 9, 6] and np.isclose(r.lse[3, 0], np.log(np.exp(0.8 * np.tanh(
        0.3 * np.concatenate([kc[p] for p in table[1]], axis=1)[0, :6] @ q[3, 0] / 0.8)).sum()))
    r = moves.paged_attention(q, kc, vc, table, lens, starts, 0.0, slopes=[0.5] * 4, window=3, prefix=[1, 0])
    w = np.exp(-0.5 * np.array([7, 2, 1, 0]))
    assert np.isclose(r.lse[0, 2], np.log(w.sum()))


def scores(**kw):
    a = dict(softcap=0.0, window=0, slopes=None, prefix_lens=None, tree_mask=None, mask_stride=1, mask_words=1)
    a.update(kw)
    return fa.PagedScores(**a)


def attend(sc, c=None, b=None, causal=True, scale=0.1, ws=P, nbytes=1 << 30, path=0):
    return fa.fa_fwd_paged_ex(c or cache(), b or batch(), sc, P, P, P, 4, fa.PagedStrides(512, 128, 512, 128), 2, path, scale, causal,
                              ws, nbytes, None)


def test_scores_that_are_refused():
    for kw in (dict(window=-1), dict(tree_mask=P, mask_words=0), dict(tree_mask=P, mask_words=65, mask_stride=65),
               dict(tree_mask=P, mask_words=2, mask_stride=1), dict(tree_mask=P, mask_stride=(1 << 40) + 1)):
        assert attend(scores(**kw)) == SHAPE, kw
    for kw in (dict(tree_mask=P, window=3), dict(tree_mask=P, slopes=P), dict(tree_mask=P, prefix_lens=P), dict(tree_mask=P + 2),
               dict(slopes=P + 1), dict(prefix_lens=P + 2)):
        assert attend(scores(**kw)) == UNSUPPORTED, kw
    assert attend(scores(tree_mask=P), causal=False) == UNSUPPORTED
    for cap in (-1.0, float("nan"), float("inf"), 1025.0):
        assert attend(scores(softcap=cap)) == fa.FA_ERR_BAD_SCALE, cap
    # As fa_fwd_paged otherwise.
    for sc in (None, scores(), scores(softcap=3.0), scores(tree_mask=P), scores(window=5)):
        assert attend(sc, scale=float("inf")) == fa.FA_ERR_BAD_SCALE and attend(sc, path=3) == UNSUPPORTED
        assert attend(sc, cache(K=None)) == NULL and attend(sc, cache(d_v=64)) == UNSUPPORTED
        assert attend(sc, b=batch(T=0)) == fa.FA_OK
        long = batch(max_blocks=256, table_stride=256)
        need = fa.fa_fwd_paged_ex_workspace_bytes(3, 5, 4096, 4, 2, 128, 128, 0, 2)
        assert need > 0 and attend(sc, b=long, nbytes=1024) == fa.FA_ERR_WORKSPACE and attend(sc, b=long, ws=None) == fa.FA_ERR_WORKSPACE
    assert fa.fa_fwd_paged_ex_workspace_bytes(3, 5, 4096, 4, 2, 96, 128, 0, 2) == 0
    assert ctypes.sizeof(fa.PagedScores) == 8 + 3 * 8 + 8 + 8


def test_score_arguments_that_are_refused():
    from paper_2609_21264_amd import _scores

    for kw in (dict(softcap=0.0), dict(softcap=-2), dict(softcap=2000.0), dict(window=0), dict(window=-1), dict(window=1 << 31)):
        a = dict(softcap=None, slopes=None, window=None, prefix_lens=None, tree_mask=None)
        a.update(kw)
        with pytest.raises(ValueError, match="softcap must be|window must be"):
            _scores(*a.values(), 3, 4, 1, 0)
    with pytest.raises(ValueError, match="slopes must be a contiguous"):
        _scores(None, torch.zeros(3), None, None, None, 3, 4, 1, 0)
    with pytest.raises(ValueError, match="slopes must be on"):
        _scores(None, torch.zeros(4), None, None, None, 3, 4, 1, 0)
    with pytest.raises(ValueError, match="1-d int32"):
        _scores(None, None, None, torch.zeros(1), None, 3, 4, 1, 0)
    with pytest.raises(ValueError, match="must be on the device"):
        _scores(None, None, None, None, torch.zeros(3, 1, dtype=torch.int32), 3, 4, 1, 0)
