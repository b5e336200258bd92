"""Paged attention with forms where the kernel for many rows splits blocks over workgroups on the device, and where there are
more sequences than a wave has lanes; bars as in test_gpu_paged_forms.py. That blocks are split is asserted on the host, by the
rule that the kernel goes by."""

import pytest
import torch

import paper_2609_21264_amd as fa
from paged import Batch
from test_gpu_cache_moves import tree_parents
from test_gpu_paged_forms import DIMS, PATHS, check, slopes_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)
NEW, KEYS = [1, 2, 200], [9000, 3000, 6000]


def is_split(bt, causal=True, window=None, prefix_lens=None, tree_mask=None, **_):
    """Whether blocks of the kernel for many rows are split: 4 units and one per 64 keys that its rows may see a block, shared by
    512 workgroups (blocks of 128 row-heads; d_qk = 192 and e4m3 256 of 256)."""
    short = not bt.fp8 and bt.dqk != 192
    cols, wgs, group = (128, 512, bt.Hq // bt.Hkv) if short else (256, 256, bt.Hq // bt.Hkv)
    total = longest = most = 0
    for b, (n, kv) in enumerate(zip(bt.new, bt.keys)):
        pre = 0 if prefix_lens is None else min(max(int(prefix_lens[b]), 0), kv)
        for c0 in range(0, n * group, cols):
            p0, p1 = kv - n + c0 // group, kv - n + (min(c0 + cols, n * group) - 1) // group
            end = kv
            if tree_mask is None and (causal or window):
                end = max(min(kv, p1 + 1 if causal else p1 + window), pre)
            tiles = -(-end // 64)
            if window:
                tiles -= max(min(max(p0 - window + 1, 0) // 64, tiles) - -(-pre // 64), 0)
            total += (4 + tiles) * bt.Hkv
            longest = max(longest, 4 + tiles)
            most += bt.Hkv
    per = max(8, (total - 1) // wgs + 1)
    return most < wgs and longest - per > 32 and 10 * longest >= 19 * per


def forms_of(name, bt):
    pre = torch.tensor([700, 5, 333][:len(bt.new)], **I32)
    return {
        "cap": dict(softcap=20.0), "slopes": dict(slopes=slopes_of(bt.Hq)), "window": dict(window=4100), "prefix": dict(prefix_lens=pre),
        "sinks": dict(window=3001, prefix_lens=torch.tensor([4, 130, 64][:len(bt.new)], **I32)),
        "all": dict(softcap=5.0, slopes=slopes_of(bt.Hq), window=4500, prefix_lens=pre),
        "both": dict(softcap=9.0, slopes=slopes_of(bt.Hq)),
        "steep": dict(slopes=torch.tensor([1e7, 300.0, 40.0, -1e6], device=DEV)),
    }[name]


@pytest.mark.parametrize("form", ["cap", "slopes", "window", "prefix", "sinks", "all", "both", "steep"])
@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_split_blocks(form, dims, fp8):
    bt = Batch(NEW, KEYS, 4, 1, *dims, 16, fp8, seed=3)
    for causal in (True, False):
        kw = dict(forms_of(form, bt), causal=causal)
        assert is_split(bt, **kw)
        o, lse = bt.attend(scale=0.09, return_lse=True, path="many", **kw)
        check(bt, o, lse, 0.09, what=f"causal={causal}", **kw)


@pytest.mark.parametrize("cap", [None, 7.0])
@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_split_trees(cap, dims, fp8):
    """Trees whose masks lie in a block's last part, over cached keys in the parts before."""
    sizes = [60, 64, 7]
    bt = Batch(sizes, [9060, 4000, 1500], 4, 1, *dims, 16, fp8, seed=4)
    mask, _ = fa.tree_mask(torch.tensor(sum((tree_parents(n, n) for n in sizes), []), **I32), bt.d_q_starts, bt.d_kv_lens, words=2)
    kw = dict(tree_mask=mask, softcap=cap)
    assert is_split(bt, **kw)
    o, lse = bt.attend(scale=0.09, return_lse=True, path="many", **kw)
    check(bt, o, lse, 0.09, **kw)


@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_split_blocks_without_some_pages(dims, fp8):
    """Pages that are not there in the first, the middle and the last part, and whole parts of them."""
    bt = Batch([60, 200], [9000, 6000], 4, 1, *dims, 16, fp8, seed=5)
    bt.table[0, 0], bt.table[0, 200:300], bt.table[1, 7], bt.table[1, 370:375] = -1, bt.n_pages, 1 << 30, -9
    bt._to(DEV, "hnd")
    mask, _ = fa.tree_mask(torch.tensor(sum((tree_parents(n, n) for n in bt.new), []), **I32), bt.d_q_starts, bt.d_kv_lens, words=7)
    for kw in (dict(forms_of("cap", bt)), dict(forms_of("slopes", bt)), dict(forms_of("sinks", bt)), dict(forms_of("both", bt)),
               dict(tree_mask=mask)):
        assert is_split(bt, **kw)
        o, lse = bt.attend(scale=0.09, return_lse=True, path="many", **kw)
        check(bt, o, lse, 0.09, what=str(list(kw)), **kw)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("form", ["prefix", "sinks", "slopes", "tree"])
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_more_sequences_than_lanes(path, form, fp8):
    """150 sequences of 0, 1, 5 and 40 new tokens with a prefix each, a long one behind the first 64 and the first 128; without
    a path both kernels have work."""
    new = [(0, 1, 5, 40)[(7 * b + b // 5) % 4] for b in range(150)]
    keys = [n + (37 * b) % 90 for b, n in enumerate(new)]
    new[97], keys[97], new[140], keys[140], new[149], keys[149] = 300, 5000, 1, 2500, 3, 70
    bt = Batch(new, keys, 8, 4, 64, 64, 16, fp8, seed=6, extra=1)
    prefix = torch.tensor([(13 * b) % (k + 4) for b, k in enumerate(keys)], **I32)
    kw = {"prefix": dict(prefix_lens=prefix, softcap=11.0), "sinks": dict(prefix_lens=prefix, window=50),
          "slopes": dict(slopes=slopes_of(8), prefix_lens=prefix), "tree": {}}[form]
    if form == "tree":
        parents = sum((tree_parents(n, b) for b, n in enumerate(new)), []) + [-1]
        kw["tree_mask"], _ = fa.tree_mask(torch.tensor(parents, **I32), bt.d_q_starts, bt.d_kv_lens, words=10)
    elif form != "sinks":  # items of 64 row-heads of the sequences with more than 32, 6 units and one per 128 keys
        units = sum(-(-2 * n // 64) * 4 * (6 + (2 * k - n) // 256) for n, k in zip(new, keys) if 2 * n > 32)
        assert units >= 2750
    o, lse = torch.full((bt.T, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((bt.T, 8), 7.0, device=DEV)
    bt.attend(scale=0.11, out=o, lse=lse, path=path, **kw)
    assert bool((o[-1] == 7).all()) and bool((lse[-1] == 7).all())
    check(bt, o, lse, 0.11, what=f"{path}", **kw)
