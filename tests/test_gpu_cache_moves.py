"""Positions of several axes, drafted trees, and moves in the paged cache on the GPU, against whole numbers and float64.

Tolerance of a turned element, as in tests/paged.py: fp32 products and sums of a pair, 2^-22 (|x| + |y|), and one rounding
to bf16 (2^-8 of the value) or e4m3 (2^-4, 2^-10 absolute below its smallest normal value).
"""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import moves
from paged import BF16, E4M3, Batch, cos_sin_table, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def near(got, want, size, rel=2.0 ** -8, least=0.0):
    off = np.abs(got - want) - (rel * np.abs(want) + 2.0 ** -22 * size + least)
    assert off.max(initial=-1) <= 0, f"off by {np.abs(got - want).max():.3e}"


def positions_of(T, axes, n_pos, seed=0):
    return torch.randint(0, n_pos, (T, axes), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


def axes_of(pairs, axes, how, seed=0):
    if how == "sections":
        return torch.tensor([c * axes // pairs for c in range(pairs)], dtype=torch.uint8)
    if how == "cyclic":
        return torch.tensor([c % axes for c in range(pairs)], dtype=torch.uint8)
    return torch.randint(0, axes, (pairs,), generator=torch.Generator().manual_seed(seed), dtype=torch.uint8)


ROTATIONS = [  # B, H, S, d, rot, begin, inter, axes, how
    (1, 1, 1, 64, 64, 0, False, 1, "none"), (2, 3, 37, 64, 64, 0, True, 3, "sections"), (1, 4, 129, 128, 128, 0, False, 3, "sections"),
    (3, 2, 50, 128, 64, 64, False, 3, "cyclic"), (1, 5, 33, 192, 64, 128, True, 2, "random"), (2, 2, 20, 192, 32, 8, False, 4, "random"),
    (1, 2, 300, 8, 8, 0, True, 1, "none"), (1, 1, 7, 1024, 1024, 0, False, 3, "cyclic"), (2, 7, 65, 72, 48, 16, False, 3, "sections"),
    (1, 2, 9, 64, 0, 0, False, 1, "none"),
]


@pytest.mark.parametrize("case", ROTATIONS, ids=str)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate(case, inverse):
    B, H, S, d, rot, begin, inter, axes, how = case
    g = torch.Generator().manual_seed(S)
    x, n_pos = torch.randn(B, H, S, d, generator=g).to(BF16), 77
    table = cos_sin_table(n_pos if how != "none" else max(S, n_pos), rot, 3) if rot else torch.zeros(S, 0)
    pos = pa = None
    if how != "none":
        pos = positions_of(B * S, axes, n_pos, 4).view(B, S, axes)
        pa = axes_of(rot // 2, axes, how, 5)
    kw = dict(positions=None if pos is None else pos.to(DEV), pair_axes=None if pa is None else pa.to(DEV), rot_begin=begin,
              interleaved=inter, inverse=inverse)
    y = fa.rotate(x.to(DEV), table.to(DEV), **kw)
    want = np.zeros((B, H, S, d))
    for b in range(B):
        for s in range(S):
            rows = moves.rows_of(pos[b, s].tolist() if pos is not None else [s], pa, rot // 2, len(table))
            want[b, :, s] = moves.rotate_at(f64(x)[b, :, s], f64(table), rows, begin, inter, -1.0 if inverse else 1.0)
    size = 2 * np.abs(f64(x)).max()
    near(f64(y), want, size)
    assert torch.equal(y[..., :begin].cpu(), x[..., :begin]) and torch.equal(y[..., begin + rot:].cpu(), x[..., begin + rot:])
    # Packed rows, other strides, and in place: the same bits.
    wide = torch.zeros(B, S, H + 1, d + 8, dtype=BF16, device=DEV)
    view = wide[:, :, :H, :d].permute(0, 2, 1, 3)
    view.copy_(x)
    assert torch.equal(fa.rotate(view, table.to(DEV), out=view, **kw), y) and view is not None
    assert torch.equal(view, y) and float(wide[:, :, H].abs().max()) == 0
    if B == 1:
        packed = x[0].transpose(0, 1).contiguous().to(DEV)
        kw["positions"] = None if pos is None else pos[0].to(DEV)
        assert torch.equal(fa.rotate(packed, table.to(DEV), **kw).transpose(0, 1), y[0])


def test_rotate_gradient():
    """The inverse is the adjoint: <R x, w> = <x, R' w>, within the roundings to bf16 of R x and R' w; and differences of the
    (linear) rotation in float64 are its values."""
    g = torch.Generator().manual_seed(0)
    x, w = (torch.randn(2, 3, 41, 64, generator=g).to(BF16) for _ in range(2))
    table, pos, pa = cos_sin_table(50, 64), positions_of(82, 3, 50).view(2, 41, 3), axes_of(32, 3, "cyclic")
    kw = dict(positions=pos.to(DEV), pair_axes=pa.to(DEV))
    y, dx = fa.rotate(x.to(DEV), table.to(DEV), **kw), fa.rotate(w.to(DEV), table.to(DEV), inverse=True, **kw)
    bar = 2.0 ** -8 * ((np.abs(f64(y)) * np.abs(f64(w))).sum() + (np.abs(f64(x)) * np.abs(f64(dx))).sum()) * 1.01
    assert abs((f64(y) * f64(w)).sum() - (f64(x) * f64(dx)).sum()) <= bar
    # Along one direction: (R(x + h e) - R(x)) / h with h = 1 in one element, exact in bf16 inputs of small whole numbers.
    xi = torch.randint(-3, 4, (2, 3, 41, 64), generator=g).to(BF16)
    e = torch.zeros_like(xi)
    e[1, 2, 17, 5] = 1
    d = f64(fa.rotate((xi + e).to(DEV), table.to(DEV), **kw)) - f64(fa.rotate(xi.to(DEV), table.to(DEV), **kw))
    col = f64(fa.rotate(e.to(DEV), table.to(DEV), **kw))
    assert np.abs(d - col).max() <= 2.0 ** -8 * (2 * 3 * 2 ** 0.5 + 3)  # roundings of values up to 3 sqrt 2, 3 sqrt 2 + 1 and 1
    assert np.abs((d * f64(w)).sum() - f64(dx)[1, 2, 17, 5]) <= 2.0 ** -8 * 12 * np.abs(f64(w)[1, 2, 17]).sum()


APPENDS = [  # new, keys, Hq, Hkv, dqk, dv, page, fp8, rot, begin, inter, axes, how
    ([1], [1], 4, 2, 64, 64, 16, False, 64, 0, False, 1, "none"), ([26], [90], 8, 2, 128, 128, 16, False, 128, 0, False, 1, "none"),
    ([5, 0, 17], [40, 9, 17], 4, 4, 128, 128, 32, True, 128, 0, False, 3, "sections"),
    ([33, 3], [70, 3], 7, 1, 64, 64, 16, False, 32, 16, True, 3, "cyclic"), ([40], [55], 6, 2, 192, 128, 64, True, 64, 128, False, 2, "random"),
]


@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append_at_positions(case):
    new, keys, Hq, Hkv, dqk, dv, page, fp8, rot, begin, inter, axes, how = case
    bt = Batch(new, keys, Hq, Hkv, dqk, dv, page, fp8, extra=2)
    n_pos = 61
    table, pos = cos_sin_table(n_pos, rot), positions_of(bt.T, axes, n_pos)
    pos[0, 0] = -5
    pos[-3, -1] = n_pos + 4  # both count as the table's ends
    pa = None if how == "none" else axes_of(rot // 2, axes, how)
    before_k, before_v = bt.d_k_cache.clone(), bt.d_v_cache.clone()
    q_out = torch.full_like(bt.d_q, 7)
    dpos = (pos if axes > 1 else pos[:, 0]).to(DEV)
    if axes > 1:
        dpos = dpos.t().contiguous().t()  # axis by axis
    bt.append(q=bt.d_q, q_out=q_out, cos_sin=table.to(DEV), rot_begin=begin, interleaved=inter, positions=dpos,
              pair_axes=None if pa is None else pa.to(DEV))
    torch.cuda.synchronize()
    kc, vc = bt.values(bt.d_k_cache, bt.k_scale), bt.values(bt.d_v_cache, bt.v_scale)
    touched = np.zeros(kc.shape[:1] + kc.shape[2:3], dtype=bool)
    rel = 2.0 ** -4 if fp8 else 2.0 ** -8
    for b, (n, kv) in enumerate(zip(new, keys)):
        for i in range(n):
            t, key = int(bt.q_starts[b]) + i, kv - n + i
            rows = moves.rows_of(pos[t].tolist(), pa, rot // 2, n_pos)
            k, q = (moves.rotate_at(f64(x)[t], f64(table), rows, begin, inter) for x in (bt.k, bt.q))
            near(f64(q_out)[t], q, 2 * np.abs(f64(bt.q)[t]).max())
            pg, slot = int(bt.table[b, key // page]), key % page
            touched[pg, slot] = True
            # (e4m3: the quotient by the scale is rounded to fp32 first, 2^-24, and small values have steps of 2^-9.)
            for got, want, sc in ((kc, k, bt.k_scale), (vc, f64(bt.v)[t], bt.v_scale)):
                least = f64(sc)[:, None] * 2.0 ** -10 * 1.01 if fp8 else 0.0
                clip = 448 * f64(sc)[:, None] if fp8 else np.inf
                near(got[pg, :, slot], np.clip(want, -clip, clip), 4 * np.abs(want).max() + 8, rel, least)
    assert torch.equal(q_out[-2:], torch.full_like(q_out[-2:], 7))
    raw = torch.uint8 if fp8 else torch.int16
    for now, was in ((bt.d_k_cache, before_k), (bt.d_v_cache, before_v)):
        same = (now.view(raw) == was.view(raw)).permute(0, 2, 1, 3).flatten(2).all(2).cpu().numpy()
        assert same[~touched].all()


def test_append_at_the_places_is_the_append():
    """Positions that are the tokens' places, by one axis and by three alike, give the same bits as none."""
    for fp8 in (False, True):
        a, b, c = (Batch([3, 9], [40, 9], 8, 2, 128, 128, 16, fp8, seed=1) for _ in range(3))
        table = cos_sin_table(64, 128).to(DEV)
        pos = torch.tensor([37, 38, 39] + list(range(9)), dtype=torch.int32, device=DEV)
        outs = [a.append(q=a.d_q, cos_sin=table), b.append(q=b.d_q, cos_sin=table, positions=pos),
                c.append(q=c.d_q, cos_sin=table, positions=pos[:, None].expand(-1, 3),
                         pair_axes=(torch.arange(64, device=DEV) % 3).to(torch.uint8))]
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        for x in (b, c):
            assert torch.equal(a.d_k_cache.view(torch.uint8), x.d_k_cache.view(torch.uint8))
            assert torch.equal(a.d_v_cache.view(torch.uint8), x.d_v_cache.view(torch.uint8))


def tree_parents(n, seed, kind="random"):
    g = torch.Generator().manual_seed(seed)
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "roots":
        return [-1] * n
    return [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)]


@pytest.mark.parametrize("sizes,words,kind", [([1], 1, "random"), ([26], 1, "random"), ([60, 0, 7, 64], 2, "random"), ([33] * 5, 2, "chain"),
                                              ([70], 2, "random"), ([64], 3, "chain"), ([2048], 64, "random"), ([2500, 3], 5, "chain"),
                                              ([9] * 300, 1, "roots"), ([4096, 31], 64, "random"), ([4096], 2, "chain"),
                                              ([97, 32, 31, 33, 64, 65], 4, "random")], ids=str)
def test_tree_mask(sizes, words, kind):
    parents = [tree_parents(n, i, kind) for i, n in enumerate(sizes)]
    starts, lens = [2], []
    for i, n in enumerate(sizes):
        starts.append(starts[-1] + n)
        lens.append(n + 11 * i)
    flat = [5, -1] + sum(parents, []) + [0]
    wrong = starts[0] + sizes[0] - 1
    if sizes[0] > 2:  # a parent that is none: itself
        flat[wrong] = parents[0][-1] = sizes[0] - 1
    i32 = dict(dtype=torch.int32, device=DEV)
    mask, positions = torch.full((len(flat), words + 1), 9, **i32), torch.full((len(flat),), 9, **i32)
    got = fa.tree_mask(torch.tensor(flat, **i32), torch.tensor(starts, **i32), torch.tensor(lens, **i32), words=words,
                       mask=mask[:, :words], positions=positions)
    assert got[1] is positions
    m, at = mask.cpu().numpy(), positions.cpu().numpy()
    assert (m[:, words] == 9).all() and (m[:2] == 9).all() and (m[-1] == 9).all() and (at[[0, 1, -1]] == 9).all()
    m = m[:, :words].astype(np.uint32)
    for b, n in enumerate(sizes):
        for i, path in enumerate(moves.paths(parents[b])):
            t = starts[b] + i
            want = [sum(1 << (j & 31) for j in path if j >> 5 == w) for w in range(words)]
            assert m[t].tolist() == want, (b, i)
            assert at[t] == lens[b] - n + len(path) - 1


def test_tree_mask_of_too_long_a_sequence():
    """Nothing is written for it, and the others have their rows."""
    i32 = dict(dtype=torch.int32, device=DEV)
    parents = torch.full((4097 + 3,), -1, **i32)
    parents[4098:] = torch.tensor([0, 0])
    mask, pos = torch.full((4100, 1), 9, **i32), torch.full((4100,), 9, **i32)
    fa.tree_mask(parents, torch.tensor([0, 4097, 4100], **i32), torch.tensor([5000, 10], **i32), mask=mask, positions=pos)
    assert bool((mask[:4097] == 9).all()) and bool((pos[:4097] == 9).all())
    assert mask[4097:, 0].tolist() == [1, 3, 5] and pos[4097:].tolist() == [7, 8, 8]


def test_outputs_that_overlap_are_refused():
    i32 = dict(dtype=torch.int32, device=DEV)
    buf = torch.zeros(64, **i32)
    starts, lens = torch.tensor([0, 5], **i32), torch.tensor([9], **i32)
    with pytest.raises(ValueError, match="positions must not overlap parents"):
        fa.tree_mask(buf[:5], starts, lens, positions=buf[4:9])
    with pytest.raises(ValueError, match="mask must not overlap parents"):
        fa.tree_mask(buf[:5], starts, lens, mask=buf[:10:2, None])
    with pytest.raises(ValueError, match="positions must not overlap mask"):
        fa.tree_mask(buf[:5], starts, lens, mask=buf[10:15, None], positions=buf[12:17])
    fa.tree_mask(buf[:5], starts, lens, mask=buf[10:15, None], positions=buf[15:20])
    bt = Batch([3], [20], 2, 2, 64, 64, 16)
    kept = torch.tensor([[0]], **i32)
    with pytest.raises(ValueError, match="new_lens must not overlap kv_lens"):
        fa.kv_compact(bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.d_kv_lens, bt.d_q_starts, kept, kept[0], new_lens=bt.d_kv_lens)
    x = torch.zeros(1, 4, 9, 64, dtype=BF16, device=DEV)
    with pytest.raises(ValueError, match="x itself or lie before or behind"):
        fa.rotate(x[:, :3], torch.zeros(9, 64, device=DEV), out=x[:, 1:])
    with pytest.raises(ValueError, match="rows of out overlap"):
        fa.rotate(x, torch.zeros(9, 64, device=DEV), out=torch.zeros(1, 1, 9, 64, dtype=BF16, device=DEV).expand(1, 4, 9, 64))


def test_rotate_many_heads():
    """More heads than a dimension of the grid has workgroups for."""
    g = torch.Generator().manual_seed(3)
    x, table = torch.randn(2, 600001, 1, 8, generator=g).to(BF16), cos_sin_table(4, 8)
    y = f64(fa.rotate(x.to(DEV), table.to(DEV), interleaved=True))
    c, s = f64(table)[0, :4], f64(table)[0, 4:]
    a, b = f64(x)[..., 0::2], f64(x)[..., 1::2]
    near(y[..., 0::2], a * c - b * s, 10.0)
    near(y[..., 1::2], b * c + a * s, 10.0)


COMPACTS = [  # new, keys, kept, heads, dqk, dv, page, fp8, order
    ([5], [5], [[1, 3, 4]], 2, 64, 64, 16, False, "hnd"), ([60, 3, 0, 20], [77, 3, 9, 20], [[0, 2, 3, 17, 18, 59], [], [], list(range(20))], 8, 128, 128, 16, False, "hnd"),
    ([40, 64], [400, 64], [list(range(1, 38)), list(range(0, 64, 2))], 3, 192, 128, 32, True, "nhd"),
    ([33] * 40, [50] * 40, [[(i + 3 * b) % 33 for i in range(1)] for b in range(40)], 6, 64, 64, 64, True, "hnd"),
    ([17], [200], [[16]], 1, 128, 128, 128, False, "nhd"),
]


@pytest.mark.parametrize("case", COMPACTS, ids=lambda c: f"{len(c[0])}x{c[0][0]}-{c[3]}-{c[4]}-{c[6]}-{c[7]}-{c[8]}")
def test_compact(case):
    new, keys, kept, heads, dqk, dv, page, fp8, order = case
    bt = Batch(new, keys, heads, heads, dqk, dv, page, fp8, order=order)
    most = max(len(k) for k in kept) + 2
    rows = torch.tensor([k + [-9] * (most - len(k)) for k in kept], dtype=torch.int32)
    n = torch.tensor([len(k) for k in kept], dtype=torch.int32)
    raw = torch.uint8 if fp8 else torch.int16
    want = [moves.compact(c.view(raw).numpy(), bt.table.tolist(), keys, bt.q_starts.tolist(), kept, n.tolist())
            for c in (bt.k_cache, bt.v_cache)]
    lens = fa.kv_compact(bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.d_kv_lens, bt.d_q_starts, rows.to(DEV), n.to(DEV))
    assert lens.tolist() == want[0][1]
    for got, (w, _) in zip((bt.d_k_cache, bt.d_v_cache), want):
        assert np.array_equal(got.cpu().view(raw).numpy(), w)


def test_compact_odd_arrays():
    """Numbers that are none, more kept than new, more new than keys, a page that is not there: what is left moves, and lengths
    stay within what there is."""
    bt = Batch([6, 6, 6, 4], [40, 40, 40, 9], 2, 2, 64, 64, 16)
    bt.table[1, 40 // 16] = bt.n_pages
    bt.kv_lens[3] = 2  # more new tokens than keys
    bt._to(DEV, "hnd")
    rows = torch.tensor([[2, -1, 77, 5], [1, 2, 3, 4], [1, 2, 4, 5], [3, 3, 3, 3]], dtype=torch.int32)
    n = torch.tensor([4, 3, 1000, -3], dtype=torch.int32)
    want = [moves.compact(c.view(torch.int16).numpy(), bt.table.tolist(), bt.kv_lens.tolist(), bt.q_starts.tolist(), rows.tolist(),
                          n.tolist()) for c in (bt.k_cache, bt.v_cache)]
    lens = fa.kv_compact(bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.d_kv_lens, bt.d_q_starts, rows.to(DEV), n.to(DEV))
    assert lens.tolist() == want[0][1] == [38, 37, 38, 0]
    for got, (w, _) in zip((bt.d_k_cache, bt.d_v_cache), want):
        assert np.array_equal(got.cpu().view(torch.int16).numpy(), w)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,page,n,layout", [(1, 16, 1, "hnd"), (3, 32, 40, "nhd"), (8, 64, 7, "layers"), (5, 128, 3, "gaps"), (2, 16, 300, "hnd")])
def test_copy(dqk, dv, fp8, heads, page, n, layout):
    total = 2 * n + 5
    raw = torch.uint8 if fp8 else torch.int16
    g = torch.Generator().manual_seed(n)
    caches, wholes = [], []
    for d in (dqk, dv):
        shape = {"hnd": (total, heads, page, d), "nhd": (total, page, heads, d), "layers": (total, heads, page, d),
                 "gaps": (total, heads + 1, page + 1, d + 16)}[layout]
        whole = torch.randint(0, 127, shape, generator=g, dtype=torch.int32).to(raw).to(DEV)
        view = whole.permute(0, 2, 1, 3) if layout == "nhd" else whole[:, :heads, :page, :d]
        if layout == "layers":
            view = whole.view(total, 2, heads // 2, page, d).flatten(1, 2)
        caches.append(view)
        wholes.append(whole)
    order = torch.randperm(total, generator=g).to(torch.int32)
    src, dst = order[:n + 3].clone(), order[n:2 * n + 3].clone()
    src[n:], dst[n:] = torch.tensor([-1, int(order[0]), int(order[1])]), torch.tensor([int(order[2 * n + 4]), total, int(order[1])])
    want = [w.clone() for w in wholes]
    for c, w in zip(caches, want):
        wc = w.as_strided(c.shape, c.stride())
        wc[dst[:n].long()] = c[src[:n].long()]
    k, v = (c.view(E4M3 if fp8 else BF16) for c in caches)
    assert fa.kv_copy(k, v, src.to(DEV), dst.to(DEV)) is None
    for w, x in zip(wholes, want):
        assert torch.equal(w, x)


def test_far_pages():
    """Pages and heads behind 2^32 bytes: copied and closed up exactly."""
    heads, page, d = 64, 128, 128
    pages = (1 << 32) // (heads * page * d * 2) + 9
    k = torch.zeros(pages, heads, page, d, dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator(device=DEV).manual_seed(0)
    for c in (k, v):
        c[-3:].normal_(generator=g)
        c[0].normal_(generator=g)
    i32 = dict(dtype=torch.int32, device=DEV)
    was = k[0].clone(), v[0].clone()
    fa.kv_copy(k, v, torch.tensor([0], **i32), torch.tensor([pages - 4], **i32))
    assert torch.equal(k[pages - 4], was[0]) and torch.equal(v[pages - 4], was[1])
    table = torch.tensor([[pages - 2, pages - 1]], **i32)
    want = k[pages - 1, :, 2].clone(), v[pages - 1, :, 2].clone()
    fa.kv_compact(k, v, table, torch.tensor([133], **i32), torch.tensor([0, 6], **i32), torch.tensor([[3]], **i32),
                  torch.tensor([1], **i32))
    assert torch.equal(k[pages - 2, :, 127], want[0]) and torch.equal(v[pages - 2, :, 127], want[1])


def test_streams_and_graphs():
    """All calls of one step captured in a graph and on another stream: every replay as the eager calls, with other
    arrays in place and eager work between."""
    bt = Batch([9, 26], [60, 300], 8, 2, 128, 128, 16)
    i32 = dict(dtype=torch.int32, device=DEV)
    table = cos_sin_table(400, 128).to(DEV)
    parents = torch.tensor(tree_parents(9, 1) + tree_parents(26, 2), **i32)
    kept, n_kept = torch.tensor([[0, 4, 7], [0, 11, 25]], **i32), torch.tensor([3, 2], **i32)
    src, dst = torch.tensor([1, 3], **i32), torch.tensor([int(bt.n_pages) - 1, -1], **i32)
    x, y = bt.d_q.clone(), torch.empty_like(bt.d_q)

    def step():
        mask, pos = fa.tree_mask(parents, bt.d_q_starts, bt.d_kv_lens)
        q = bt.append(q=bt.d_q, cos_sin=table, positions=pos)
        lens = fa.kv_compact(bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.d_kv_lens, bt.d_q_starts, kept, n_kept)
        fa.kv_copy(bt.d_k_cache, bt.d_v_cache, src, dst)
        fa.rotate(x, table, positions=pos, out=y)
        return mask, pos, q, lens

    start = bt.d_k_cache.clone(), bt.d_v_cache.clone()

    def reset():
        bt.d_k_cache.copy_(start[0])
        bt.d_v_cache.copy_(start[1])

    def held(outs):
        torch.cuda.synchronize()
        return [t.clone().view(torch.uint8) for t in (*outs, bt.d_k_cache, bt.d_v_cache, y)]

    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        outs = step()
    for turn in range(3):
        if turn:
            parents.copy_(torch.tensor(tree_parents(9, 5 + turn) + tree_parents(26, 7 + turn), **i32))
            kept.add_(torch.tensor([[0, 1, 1], [0, 2, 0]], **i32) * (turn == 1))
        reset()
        want = held(step())
        reset()
        graph.replay()
        got = held(outs)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        reset()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        assert all(torch.equal(a, b) for a, b in zip(held(other), want))
    reset()
    torch.cuda.synchronize()
    # Named streams.
    mask, pos = fa.tree_mask(parents, bt.d_q_starts, bt.d_kv_lens, stream=side)
    side.synchronize()
    assert torch.equal(mask.view(torch.uint8), want[0]) and torch.equal(pos.view(torch.uint8), want[1])
    z = fa.rotate(x, table, positions=pos, stream=side.cuda_stream)
    fa.kv_copy(bt.d_k_cache, bt.d_v_cache, src, dst, stream=side)
    side.synchronize()
    assert torch.equal(z.view(torch.uint8), want[6]) and torch.equal(bt.d_k_cache[dst[0].item()], start[0][1])
