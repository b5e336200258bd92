"""Slopes up to the largest and infinite ones, on the GPU: a token sees itself alone, and the nearest of the keys that it may see."""

import pytest
import torch

from paged import Batch
from test_gpu_paged_forms import DIMS, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("path", ["few", "many"])
@pytest.mark.parametrize("dims", DIMS, ids=str)
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_slopes_without_measure(path, dims, fp8):
    """At distance 0 nothing is taken off, however steep the slope: 0 times what overflows is no number."""
    bt = Batch([130, 1, 40], [300, 500, 40], 4, 2, *dims, 16, fp8, seed=11)
    steep = torch.tensor([1e18, 1e30, 2e38, 3.4e38], device=DEV)
    for kw in (dict(), dict(softcap=20.0), dict(causal=False), dict(window=70)):
        for scale in (0.1, 1e-30, -0.1):
            o, lse = bt.attend(scale=scale, return_lse=True, path=path, slopes=steep, **kw)
            check(bt, o, lse, scale, slopes=steep, what=f"{kw} {scale}", **kw)
            alike = bt.attend(scale=scale, return_lse=True, path=path, slopes=torch.full_like(steep, float("inf")), **kw)
            same = bt.attend(scale=scale, return_lse=True, path=path, slopes=torch.full_like(steep, 3.4e38), **kw)
            assert torch.equal(alike[0], same[0]) and torch.equal(alike[1], same[1])


@pytest.mark.parametrize("path", ["few", "many"])
def test_slopes_below_zero(path):
    """The farthest key counts; far ones are not taken for infinitely far."""
    bt = Batch([130, 1], [300, 90000], 4, 2, 64, 64, 16, seed=13)
    slopes = torch.tensor([-5e17, -1e9, -3.0, 7e17], device=DEV)
    for scale in (0.1, 1e-8, 1e-12):
        o, lse = bt.attend(scale=scale, return_lse=True, path=path, slopes=slopes)
        check(bt, o, lse, scale, slopes=slopes, what=str(scale))


@pytest.mark.parametrize("path", ["few", "many"])
def test_a_slope_that_is_no_number(path):
    """Its heads' rows are O = 0 and LSE = -inf, the others as without it."""
    bt = Batch([130, 1], [300, 500], 4, 2, 128, 128, 16, seed=12)
    slopes = torch.tensor([0.1, float("nan"), 0.0, 2.0], device=DEV)
    o, lse = bt.attend(scale=0.1, return_lse=True, path=path, slopes=slopes)
    clean = bt.attend(scale=0.1, return_lse=True, path=path, slopes=slopes.nan_to_num(0.3))
    others = [0, 2, 3]
    assert torch.isneginf(lse[:, 1]).all() and not bool(o[:, 1].any())
    assert torch.equal(o[:, others], clean[0][:, others]) and torch.equal(lse[:, others], clean[1][:, others])
