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


def test_new_rows_of_a_tree_that_is_too_long():
    """A sequence of 4 097 new tokens has rows of zeros in new tensors, also where memory held something; those that
    belong to others are right."""
    parents = torch.full((4100,), -1, **I32)
    parents[4098:] = torch.tensor([0, 0], **I32)
    for _ in range(2):
        mask, positions = fa.tree_mask(parents, torch.tensor([0, 4097, 4100], **I32), torch.tensor([5000, 10], **I32))
        assert mask.shape == (4100, 64) and not bool(mask[:4097].any()) and not bool(positions[:4097].any())
        assert mask[4097:, 0].tolist() == [1, 3, 5] and not bool(mask[:, 1:].any()) and positions[4097:].tolist() == [7, 8, 8]
        held = mask.fill_(-1), positions.fill_(-1)
        torch.cuda.synchronize()
        del mask, positions, held


def test_new_rows_of_a_tree_that_is_too_long_captured():
    """The zeros are part of the captured call: every replay writes them again."""
    parents = torch.full((4100,), -1, **I32)
    starts, lens = torch.tensor([0, 4097, 4100], **I32), torch.tensor([5000, 10], **I32)
    fa.tree_mask(parents, starts, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mask, positions = fa.tree_mask(parents, starts, lens)
    for turn in range(4):
        mask.fill_(-1)
        positions.fill_(-1)
        parents[4098:] = torch.tensor([turn - 1, 1 if turn > 1 else -1], **I32)
        graph.replay()
        want, at = fa.tree_mask(parents, starts, lens)
        assert torch.equal(mask, want) and torch.equal(positions, at)
        assert not bool(mask[:4097].any()) and not bool(positions[:4097].any()) and bool(mask[4097:, 0].all())
