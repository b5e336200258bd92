"""GPU tests of the rotation and the moves around the paged cache at counts next to 2^31."""

import pytest
import torch

import paper_2609_21264_amd as fa

pytestmark = pytest.mark.gpu
BF16, DEV = torch.bfloat16, "cuda:0"


def all_equal(x, want, rows=1 << 26):
    """Whether every row of x is `want`, some rows at a time."""
    return all(bool((part == want).all()) for part in x.split(rows))


@pytest.mark.parametrize("B", [2 ** 31 - 2 ** 20, 2 ** 31 - 2 ** 20 + 1, 2 ** 31 - 1])
def test_rotate_of_very_many_batches(B):
    """As many blocks of tokens as there can be: the step from the last ones leads past 2^31. A quarter turn is exact."""
    x = torch.arange(1, 9, device=DEV).to(BF16).view(1, 1, 1, 8)
    y = torch.zeros(B, 8, dtype=BF16, device=DEV)
    table = torch.tensor([[0.0] * 4 + [1.0] * 4], device=DEV)
    fa.rotate(x.expand(B, 1, 1, 8), table, interleaved=True, out=y.view(B, 1, 1, 8))
    torch.cuda.synchronize()
    assert all_equal(y, torch.tensor([-2, 1, -4, 3, -6, 5, -8, 7], device=DEV).to(BF16))


@pytest.fixture(scope="module")
def far():
    """Arrays of 2^31 - 65 sequences, of which only the last two have new tokens: three of 20 keys, and two of 9."""
    B = 2 ** 31 - 65
    starts, lens = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    starts[-2:] = torch.tensor([3, 5], dtype=torch.int32, device=DEV)
    lens[-2:] = torch.tensor([20, 9], dtype=torch.int32, device=DEV)
    yield B, starts, lens
    del starts, lens
    torch.cuda.empty_cache()


def test_tree_mask_of_very_many_sequences(far):
    """The step from the last sequences leads past 2^31."""
    _, starts, lens = far
    parents = torch.tensor([-1, 0, 0, -1, -1], dtype=torch.int32, device=DEV)
    mask, positions = fa.tree_mask(parents, starts, lens, words=1)
    assert mask[:, 0].tolist() == [1, 3, 5, 1, 2] and positions.tolist() == [17, 18, 18, 7, 7]
