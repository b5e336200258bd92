"""What tree_mask makes when the program names no width, and of trees that are too long, on the GPU."""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import moves
from paged import Batch
from test_gpu_cache_moves import tree_parents
from test_gpu_paged_forms import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("sizes,words", [([1], 1), ([32], 1), ([33], 2), ([60, 7, 33], 4), ([9] * 30, 9), ([2048], 64), ([1500, 1200], 64)], ids=str)
def test_masks_cover_every_token_by_default(sizes, words):
    """Every token of a tree has its own bit and its ancestors', without a width or with a mask's."""
    parents = [tree_parents(n, i) for i, n in enumerate(sizes)]
    starts = torch.tensor(np.cumsum([0] + sizes).tolist(), **I32)
    args = torch.tensor(sum(parents, []), **I32), starts, torch.tensor(sizes, **I32)
    mask, positions = fa.tree_mask(*args)
    wide = torch.full((sum(sizes), 64), 9, **I32)
    assert mask.shape == (sum(sizes), words) and fa.tree_mask(*args, mask=wide)[0] is wide
    assert torch.equal(wide[:, :words], mask) and not bool(wide[:, words:].any())
    bits, at = moves.tree_bits(mask.cpu().numpy()), positions.tolist()
    for b, t0 in enumerate(starts[:-1].tolist()):
        for i, path in enumerate(moves.paths(parents[b])):
            assert set(np.flatnonzero(bits[t0 + i]).tolist()) == path and at[t0 + i] == len(path) - 1


@pytest.mark.parametrize("path", ["few", "many", None])
def test_attention_of_a_tree_of_more_than_32_tokens_by_default(path):
    bt = Batch([60, 5], [700, 90], 8, 2, 128, 128, 16)
    mask, _ = fa.tree_mask(torch.tensor(tree_parents(60, 1) + tree_parents(5, 2), **I32), bt.d_q_starts, bt.d_kv_lens)
    o, lse = bt.attend(scale=0.1, return_lse=True, tree_mask=mask, path=path)
    check(bt, o, lse, 0.1, tree_mask=mask)
    assert moves.tree_bits(mask.cpu().numpy())[range(60), range(60)].all()
