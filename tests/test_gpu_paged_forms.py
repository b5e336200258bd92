"""Attention over the paged cache with scores capped or biased, windows, prefixes and drafted trees, on the GPU against
float64.

Tolerances (half steps: bf16 2^-8 of the value, fp16 2^-11). O: P enters the product rounded, 2^-8 of it over a bf16 cache and
2^-11, or 2^-32 of the row's largest, over an e4m3 one, so O moves by that part of sum p |v|; O is rounded once, 2^-8 |O|; a
score that is off by e moves p by p e and the sum likewise (oracle.moves.Attention.off_v, off); fp32 sums, weights of joined
parts and the division add 2^-17 sum p |v|. LSE: the scores' errors weighted by p, and 2^-20 (1 + |LSE|) for sums,
logarithm and the way through log2.
"""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import moves
from paged import BF16, Batch, f64
from test_gpu_cache_moves import tree_parents

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(bt, o, lse, scale, causal=True, softcap=None, slopes=None, window=None, prefix_lens=None, tree_mask=None, what=""):
    torch.cuda.synchronize()
    ref = moves.paged_attention(f64(bt.q), bt.values(bt.k_cache, bt.k_scale), bt.values(bt.v_cache, bt.v_scale), bt.table.numpy(),
                                bt.kv_lens.tolist(), bt.q_starts.tolist(), scale, causal, softcap,
                                None if slopes is None else f64(slopes), window,
                                None if prefix_lens is None else [min(max(x, 0), k) for x, k in zip(prefix_lens.tolist(), bt.kv_lens.tolist())],
                                None if tree_mask is None else moves.tree_bits(tree_mask.cpu().numpy()))
    rows = ~np.isnan(ref.lse[:, 0])
    o, lse = f64(o)[rows], f64(lse)[rows]
    part = 2.0 ** -11 if bt.fp8 else 2.0 ** -8
    floor = (ref.keys[:, None] * 2.0 ** -32 * ref.vmax)[..., None] if bt.fp8 else 0.0
    bar = (part + 2.0 ** -17) * ref.mass + 2.0 ** -8 * np.abs(ref.o) + ref.off_v + ref.off[..., None] * ref.mass + floor + 1e-30
    lbar = ref.off + 2.0 ** -20 * (1 + np.abs(np.where(np.isneginf(ref.lse), 0, ref.lse)))
    want, wlse, bar, lbar = ref.o[rows], ref.lse[rows], (bar * 1.01)[rows], lbar[rows]
    empty = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(lse), empty), f"{what}: rows without a visible key differ"
    assert np.isfinite(o).all() and np.isfinite(lse[~empty]).all(), f"{what}: not finite"
    assert np.all(o[empty] == 0), f"{what}: O of a row without a visible key"
    off = np.abs(o - want) - bar
    assert off.max(initial=-1) <= 0, f"{what}: O off by {np.abs(o - want).max():.3e} at {np.unravel_index(off.argmax(), off.shape)}"
    loff = np.abs(lse[~empty] - wlse[~empty]) - lbar[~empty]
    assert loff.max(initial=-1) <= 0, f"{what}: LSE off by {np.abs(lse[~empty] - wlse[~empty]).max():.3e}"


DIMS = [(64, 64), (128, 128), (192, 128)]
PATHS = ["few", "many", None]


def slopes_of(hq):
    return (2.0 ** (-8.0 * (torch.arange(hq) + 1) / hq)).float().to(DEV)


def forms_of(name, bt):
    i32 = dict(dtype=torch.int32, device=DEV)
    n = len(bt.new)
    return {
        "cap": dict(softcap=20.0),
        "slopes": dict(slopes=slopes_of(bt.Hq)),
        "window": dict(window=37),
        "prefix": dict(prefix_lens=torch.tensor([(5 + 31 * b) % (k + 3) for b, k in enumerate(bt.keys)], **i32)),
        "sinks": dict(window=64, prefix_lens=torch.tensor([4] * n, **i32)),
        "all": dict(softcap=5.0, slopes=slopes_of(bt.Hq), window=90, prefix_lens=torch.tensor([17] * n, **i32)),
    }[name]


# new, keys, Hq, Hkv, page
BATCHES = {
    "tokens": ([1, 1, 1], [1, 300, 1029], 8, 2, 16),
    "drafts": ([5, 3, 0, 1], [700, 3, 9, 128], 14, 2, 32),
    "prompts": ([133, 70], [133, 400], 4, 2, 16),
    "group1": ([40, 200], [41, 640], 3, 3, 64),
}


@pytest.mark.parametrize("form", ["cap", "slopes", "window", "prefix", "sinks", "all"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_forms(form, batch, dims, fp8):
    new, keys, hq, hkv, page = BATCHES[batch]
    bt = Batch(new, keys, hq, hkv, *dims, page, fp8, seed=len(form), sigma=2.0)
    scale = 0.7 / dims[0] ** 0.5
    for causal in (True, False):
        kw = dict(forms_of(form, bt), causal=causal)
        for path in PATHS:
            o, lse = bt.attend(scale=scale, return_lse=True, path=path, **kw)
            check(bt, o, lse, scale, what=f"{path} causal={causal}", **kw)


TREES = [  # sizes, cached, Hq, Hkv, words
    ([1], [0], 4, 4, 1), ([26], [500], 8, 2, 1), ([60, 7, 0, 33], [1000, 0, 9, 31], 8, 2, 2), ([64, 64], [100, 129], 7, 1, 2),
    ([100], [77], 4, 1, 3), ([5] * 9, [40 * i for i in range(9)], 4, 2, 1), ([70, 20], [60, 333], 6, 3, 2),
]


@pytest.mark.parametrize("case", TREES, ids=str)
@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_trees(case, dims, fp8):
    sizes, cached, hq, hkv, words = case
    bt = Batch(sizes, [n + c for n, c in zip(sizes, cached)], hq, hkv, *dims, 16, fp8, seed=words, extra=2)
    parents = torch.tensor(sum((tree_parents(n, 3 * i) for i, n in enumerate(sizes)), []) + [-1, -1], dtype=torch.int32, device=DEV)
    wide = torch.full((bt.T, words + 3), -1, dtype=torch.int32, device=DEV)
    mask, _ = fa.tree_mask(parents, bt.d_q_starts, bt.d_kv_lens, words=words, mask=wide[:, :words])
    scale = dims[0] ** -0.5
    for cap in (None, 3.0):
        for path in PATHS:
            o, lse = torch.full((bt.T, hq, dims[1]), 7.0, dtype=BF16, device=DEV), torch.full((bt.T, hq), 7.0, device=DEV)
            bt.attend(scale=scale, out=o, lse=lse, path=path, tree_mask=mask, softcap=cap)
            assert float(o[-2:].float().min()) == float(o[-2:].float().max()) == 7 and float(lse[-2:].min()) == 7
            # (New tokens that have no bit are hidden.)
            check(bt, o, lse, scale, tree_mask=mask, softcap=cap, what=f"{path} cap={cap}")


def test_tree_of_a_chain_is_causal():
    """A chain sees what a causal call sees; every token alone, the cached keys and itself; a mask of zeros over no cached
    keys leaves every row empty."""
    bt = Batch([33, 12], [300, 12], 8, 2, 128, 128, 16)
    i32 = dict(dtype=torch.int32, device=DEV)
    chain, _ = fa.tree_mask(torch.tensor(tree_parents(33, 0, "chain") + tree_parents(12, 0, "chain"), **i32), bt.d_q_starts,
                            bt.d_kv_lens, words=2)
    for path in PATHS:
        o, lse = bt.attend(scale=0.1, return_lse=True, tree_mask=chain, path=path)
        bt.check(o, lse, 0.1, True, f"chain {path}")
    none = torch.zeros(45, 1, **i32)
    for path in PATHS:
        o, lse = bt.attend(scale=0.1, return_lse=True, tree_mask=none, path=path)
        check(bt, o, lse, 0.1, tree_mask=none, what=f"none {path}")
        assert torch.isneginf(lse[33:]).all() and float(o[33:].abs().max()) == 0


def test_any_mask():
    """Masks that are no trees (any bits, keys behind the words hidden), more new tokens than keys among the sequences."""
    bt = Batch([40, 70, 9], [90, 70, 30], 4, 2, 64, 64, 16)
    bt.kv_lens[2] = 4  # five of nine tokens before position 0
    bt._to(DEV, "hnd")
    g = torch.Generator().manual_seed(2)
    mask = torch.randint(-2 ** 31, 2 ** 31, (119, 2), generator=g, dtype=torch.int64).to(torch.int32).to(DEV)
    mask[5] = 0
    for path in PATHS:
        o, lse = bt.attend(scale=0.2, return_lse=True, tree_mask=mask, path=path)
        check(bt, o, lse, 0.2, tree_mask=mask, what=str(path))


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_pages_that_are_not_there(path, fp8):
    bt = Batch([30, 1, 90], [500, 700, 90], 8, 2, 128, 128, 16, fp8)
    bt.table[0, 2], bt.table[0, 30], bt.table[1, 40], bt.table[2, 0] = -1, bt.n_pages, 1 << 30, -5
    bt._to(DEV, "hnd")
    for form in ("cap", "slopes", "sinks", "prefix"):
        kw = forms_of(form, bt)
        o, lse = bt.attend(scale=0.1, return_lse=True, path=path, **kw)
        check(bt, o, lse, 0.1, what=form, **kw)
    mask, _ = fa.tree_mask(torch.tensor(sum((tree_parents(n, n) for n in bt.new), []), dtype=torch.int32, device=DEV),
                           bt.d_q_starts, bt.d_kv_lens, words=3)
    o, lse = bt.attend(scale=0.1, return_lse=True, path=path, tree_mask=mask)
    check(bt, o, lse, 0.1, tree_mask=mask, what="tree")


@pytest.mark.parametrize("form", ["cap", "window", "sinks", "slopes", "prefix"])
def test_split_over_the_chip(form):
    """Long keys of few rows, split and joined, and a chunk that is split over workgroups."""
    bt = Batch([1, 2, 600], [20000, 5000, 9000], 4, 1, 128, 128, 16, seed=3)
    kw = forms_of(form, bt)
    if "window" in kw:
        kw["window"] = 4100
    for path in PATHS:
        o, lse = bt.attend(scale=0.09, return_lse=True, path=path, **kw)
        check(bt, o, lse, 0.09, what=str(path), **kw)


@pytest.mark.parametrize("path", PATHS)
def test_windows_of_every_kind(path):
    """Windows of one key, of tiles and about them, longer than everything; prefixes at the borders of tiles, behind the keys and
    negative."""
    bt = Batch([1, 3, 140], [500, 300, 300], 4, 2, 64, 64, 16, seed=5)
    i32 = dict(dtype=torch.int32, device=DEV)
    for window in (1, 2, 63, 64, 65, 127, 128, 129, 299, 300, 2 ** 31 - 1):
        for prefix in (None, [-7, 64, 1000], [128, 0, 33]):
            for causal in (True, False):
                kw = dict(window=window, causal=causal, prefix_lens=None if prefix is None else torch.tensor(prefix, **i32))
                o, lse = bt.attend(scale=0.2, return_lse=True, path=path, **kw)
                check(bt, o, lse, 0.2, what=str(kw), **kw)


@pytest.mark.parametrize("path", ["few", "many"])
def test_steep_and_flat_scores(path):
    """Slopes so steep that only the last key counts, negative ones, scales of 0 and below, caps from tiny to the largest, scores far
    behind the cap."""
    bt = Batch([70, 2], [400, 300], 4, 2, 128, 128, 16, seed=6, sigma=3.0)
    steep = torch.tensor([40.0, 3.0, -0.5, 0.0], device=DEV)
    for scale in (0.0, -0.3, 1.0):
        for kw in (dict(slopes=steep), dict(softcap=1e-30), dict(softcap=1024.0), dict(softcap=0.5, slopes=steep), dict(softcap=30.0)):
            o, lse = bt.attend(scale=scale, return_lse=True, path=path, **kw)
            check(bt, o, lse, scale, what=f"{scale} {kw}", **kw)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("first", [255, 254, 191, 256])
def test_steep_slopes_at_the_end_of_a_tile(path, first):
    """The first row of a block stands on the last key of a tile, or about it: its own key, at distance 0, loses nothing to the
    tile's far ones."""
    for dims in DIMS:
        bt = Batch([70, 1], [first + 70, first + 1], 4, 4, *dims, 16, seed=first)
        kw = dict(slopes=torch.tensor([300.0, 40.0, 1.0, 0.01], device=DEV))
        o, lse = bt.attend(scale=0.05, return_lse=True, path=path, **kw)
        check(bt, o, lse, 0.05, what=str(dims), **kw)


@pytest.mark.parametrize("path", ["few", "many"])
def test_far_positions(path):
    """A sequence of more than 2^24 keys (many of its pages are the same few): a window with slopes is that of its end alone."""
    page, blocks = 1024, (1 << 14) + 3
    g = torch.Generator().manual_seed(4)
    i32 = dict(dtype=torch.int32, device=DEV)
    k, v = (torch.randn(8, 2, page, 64, generator=g).to(BF16).to(DEV) for _ in range(2))
    q = torch.randn(40, 4, 64, generator=g).to(BF16).to(DEV)
    table = (torch.arange(blocks, **i32) % 8)[None]
    starts, out = torch.tensor([0, 40], **i32), []
    for n, tab in ((blocks * page - 3, table), (3 * page - 3, table[:, blocks - 3:].contiguous())):
        kw = dict(slopes=torch.tensor([0.5, 0.1, 0.02, 0.0], device=DEV), window=700)
        a = fa.forward_paged(q, k, v, tab, torch.tensor([n], **i32), starts, max_q=40, return_lse=True, path=path, **kw)
        b = fa.forward_paged(q, k, v, tab, torch.tensor([n], **i32), starts, max_q=40, return_lse=True, path=path, window=300, softcap=5.0)
        out.append([*a, *b])
    for x, y in zip(*out):  # cut over the chip in other places: P rounded and sums taken in another order, on both sides
        x, y = f64(x), f64(y)
        bar = 2.0 ** -19 * (1 + np.abs(y)) if x.ndim == 2 else 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -17) * np.abs(f64(v)).max()
        assert np.all(np.abs(x - y) <= bar)


@pytest.mark.parametrize("path", ["few", "many"])
def test_pages_behind_4_gib(path):
    """The last pages of a cache of more than 2^32 bytes."""
    bt = Batch([30, 40], [100, 70], 4, 2, 64, 64, 16, seed=12)
    pages = (1 << 32) // (2 * 16 * 64 * 2) + 100
    big = [torch.empty(pages, 2, 16, 64, dtype=BF16, device=DEV) for _ in range(2)]
    for c, d in zip(big, (bt.d_k_cache, bt.d_v_cache)):
        c[pages - bt.n_pages:] = d
    table = torch.where(bt.d_table >= 0, bt.d_table + (pages - bt.n_pages), bt.d_table)
    kw = dict(window=33, prefix_lens=torch.tensor([5, 9], dtype=torch.int32, device=DEV))
    o, lse = fa.forward_paged(bt.d_q, *big, table, bt.d_kv_lens, bt.d_q_starts, max_q=40, scale=0.1, return_lse=True, path=path, **kw)
    check(bt, o, lse, 0.1, **kw)


@pytest.mark.parametrize("path", PATHS)
def test_hidden_keys_do_not_reach_rows(path):
    """An infinity or a NaN in a hidden key reaches no row; one in a visible key makes that row's sum no number: O = 0, LSE =
    -inf."""
    bt = Batch([64, 1], [300, 200], 4, 2, 128, 128, 16, seed=7)
    for b, key, val in ((0, 100, float("nan")), (0, 20, float("inf")), (1, 50, float("nan"))):
        bt.k_cache[int(bt.table[b, key // 16]), :, key % 16] = val
    bt._to(DEV, "hnd")
    clean = Batch([64, 1], [300, 200], 4, 2, 128, 128, 16, seed=7)
    kw = dict(window=130)  # key 100 is seen by row 0 (at 236): |236 - 100| = 136: by none
    o, lse = bt.attend(scale=0.1, return_lse=True, path=path, **kw)
    check(clean, o, lse, 0.1, what="window", **kw)
    kw = dict(window=138, softcap=10.0)  # rows 0 and 1 (at 236 and 237) see key 100, 136 and 137 away
    o, lse = bt.attend(scale=0.1, return_lse=True, path=path, **kw)
    oc, lc = clean.attend(scale=0.1, return_lse=True, path=path, **kw)
    assert torch.isneginf(lse[:2]).all() and float(o[:2].abs().max()) == 0
    assert torch.equal(lse[2:64], lc[2:64]) and torch.equal(o[2:64], oc[2:64])


@pytest.mark.parametrize("path", PATHS)
def test_every_key_counts(path):
    """Values that are one-hot by key: each output element is a share of the probability, so a key that is lost, or seen by a row
    that must not, shows whatever its neighbours are."""
    for kw0, keys in ((dict(window=50), 64), (dict(softcap=4.0), 64), (dict(window=40), 128), (dict(tree=True), 128)):
        n, d = 40, 128
        bt = Batch([n], [keys + n], 4, 2, 128, d, 16, seed=8)
        vc = torch.zeros_like(bt.v_cache)
        for key in range(keys + n):
            vc[int(bt.table[0, key // 16]), :, key % 16, key % d] = 1.0
        bt.v_cache = vc
        bt._to(DEV, "hnd")
        kw = dict(kw0)
        if kw.pop("tree", False):
            kw["tree_mask"], _ = fa.tree_mask(torch.tensor(tree_parents(n, 9), dtype=torch.int32, device=DEV), bt.d_q_starts,
                                              bt.d_kv_lens, words=2)
        o, lse = bt.attend(scale=0.05, return_lse=True, path=path, **kw)
        check(bt, o, lse, 0.05, what=str(kw0), **kw)


def test_nothing_set_is_the_plain_call():
    bt = Batch([1, 50], [300, 50], 8, 2, 128, 128, 16)
    plain = bt.attend(scale=0.1, return_lse=True)
    with_none = bt.attend(scale=0.1, return_lse=True, softcap=None, window=None)
    assert torch.equal(plain[0], with_none[0]) and torch.equal(plain[1], with_none[1])
    far = bt.attend(scale=0.1, return_lse=True, window=1 << 30)
    bt.check(*far, 0.1, True, "a window longer than everything")


def test_workspace_and_strides():
    """A workspace of the stated size and not a byte more, queries and outputs in wider rows, an nhd cache."""
    bt = Batch([5, 300], [3000, 4000], 8, 2, 128, 128, 32, order="nhd", seed=2)
    T, keys = bt.T, bt.table.shape[1] * 32
    wide = torch.zeros(T, 10, 136, dtype=BF16, device=DEV)
    q = wide[:, 1:9, :128]
    q.copy_(bt.d_q)
    out = torch.zeros(T, 9, 144, dtype=BF16, device=DEV)
    for path, code in ((None, 0), ("few", 1), ("many", 2)):
        need = fa.fa_fwd_paged_ex_workspace_bytes(2, T, keys, 8, 2, 128, 128, 0, 300, code)
        guard = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
        kw = dict(softcap=8.0, window=1000)
        o, lse = fa.forward_paged(q, bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.d_kv_lens, bt.d_q_starts, max_q=300, scale=0.1,
                                  return_lse=True, out=out[:, :8, :128], workspace=guard[:need], path=path, **kw)
        check(bt, o, lse, 0.1, what=str(path), **kw)
        assert bool((guard[need:] == 77).all()) and float(out[:, 8].abs().max()) == 0 and float(out[:, :, 128:].abs().max()) == 0


def test_captured_and_other_streams():
    """One captured call serves other lengths (behind 300 keys of the second sequence lie NaNs: bits are compared), masks, prefixes
    and slopes; two streams with a workspace each."""
    def same(a, b):
        return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))

    bt = Batch([26, 26], [900, 300], 8, 2, 128, 128, 16)
    i32 = dict(dtype=torch.int32, device=DEV)
    parents = torch.tensor(tree_parents(26, 1) + tree_parents(26, 2), **i32)
    mask, _ = fa.tree_mask(parents, bt.d_q_starts, bt.d_kv_lens)
    prefix, slopes = torch.tensor([100, 3], **i32), slopes_of(8)

    def calls():
        a = bt.attend(scale=0.1, return_lse=True, tree_mask=mask)
        b = bt.attend(scale=0.1, return_lse=True, window=200, prefix_lens=prefix, softcap=9.0)
        c = bt.attend(scale=0.1, return_lse=True, slopes=slopes)
        return [*a, *b, *c]

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for lens in ([900, 300], [26, 310], [700, 26]):
        bt.d_kv_lens.copy_(torch.tensor(lens))
        mask.copy_(fa.tree_mask(torch.tensor(tree_parents(26, lens[0]) + tree_parents(26, 5), **i32), bt.d_q_starts, bt.d_kv_lens)[0])
        prefix.copy_(torch.tensor([lens[1] // 2, 20]))
        slopes.mul_(0.7)
        want = [t.clone() for t in calls()]
        graph.replay()
        torch.cuda.synchronize()
        assert same(held, want)
        side = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = []
        for s in side:
            got.append(bt.attend(scale=0.1, return_lse=True, tree_mask=mask, stream=s))
        torch.cuda.synchronize()
        assert all(same(g, want) for g in got)


def test_drafting_run():
    """Three rounds of a speculative loop: trees drafted, appended at their positions, attended to, a path kept and
    closed up; at the end the cache holds the kept tokens as a plain run would have written them, and the attention of the next
    token over it is that of the plain cache."""
    g = torch.Generator().manual_seed(11)
    Hq, Hkv, d, page, B = 8, 2, 128, 16, 3
    i32 = dict(dtype=torch.int32, device=DEV)
    pages = 3 * 20
    table = torch.randperm(pages, generator=g).to(torch.int32).view(B, 20).to(DEV)
    caches = [torch.zeros(pages, Hkv, page, d, dtype=BF16, device=DEV) for _ in range(4)]
    angles = torch.arange(320.)[:, None] * 10000.0 ** (-torch.arange(64) / 64.)
    cos_sin = torch.cat([angles.cos(), angles.sin()], 1).to(DEV)
    lens = torch.tensor([37, 5, 120], **i32)
    starts = torch.tensor([0, 37, 42, 162], **i32)
    k, v = (torch.randn(162, Hkv, d, generator=g).to(BF16).to(DEV) for _ in range(2))
    for c in (caches[:2], caches[2:]):
        fa.kv_append(k, v, *c, table, lens, starts, cos_sin=cos_sin)
    for turn in range(3):
        n = 20
        starts = torch.arange(B + 1, **i32) * n
        parents = [tree_parents(n, 7 * turn + b) for b in range(B)]
        with_drafts = lens + n
        mask, pos = fa.tree_mask(torch.tensor(sum(parents, []), **i32), starts, with_drafts)
        q, k, v = (torch.randn(B * n, h, d, generator=g).to(BF16).to(DEV) for h in (Hq, Hkv, Hkv))
        q = fa.kv_append(k, v, *caches[:2], table, with_drafts, starts, q=q, cos_sin=cos_sin, positions=pos)
        o = fa.forward_paged(q, *caches[:2], table, with_drafts, starts, max_q=n, tree_mask=mask)
        paths = []
        for b in range(B):  # the path of the deepest token
            all_paths = moves.paths(parents[b])
            paths.append(sorted(max(all_paths, key=len)))
        most = max(map(len, paths))
        kept = torch.tensor([p + [-1] * (most - len(p)) for p in paths], **i32)
        new = torch.tensor([len(p) for p in paths], **i32)
        new_lens = fa.kv_compact(*caches[:2], table, with_drafts, starts, kept, new)
        assert torch.equal(new_lens, lens + new)
        # The plain run: the kept tokens alone, at their places.
        rows = torch.tensor([b * n + i for b, p in enumerate(paths) for i in p], device=DEV)
        plain_starts = torch.cat([torch.zeros(1, **i32), new.cumsum(0).to(torch.int32)])
        q0 = torch.randn(B * n, Hq, d, generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
        del q0
        fa.kv_append(k[rows].contiguous(), v[rows].contiguous(), *caches[2:], table, new_lens, plain_starts, cos_sin=cos_sin)
        lens = new_lens
        for b in range(B):
            at = torch.arange(int(lens[b]), device=DEV)
            pg, slot = table[b].long()[at // page], at % page
            for x, y in ((caches[0], caches[2]), (caches[1], caches[3])):
                assert torch.equal(x[pg, :, slot], y[pg, :, slot])
        # What a drafted token of the path saw is what it sees in the plain cache: the same keys, so the same attention but for
        # the order of sums.
        op = fa.forward_paged(q[rows].contiguous(), *caches[2:], table, new_lens, plain_starts, max_q=most)
        bar = 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -16) * float(caches[3].abs().max())
        assert float((op.float() - o[rows].float()).abs().max()) <= bar
