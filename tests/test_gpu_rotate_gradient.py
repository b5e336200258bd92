"""The gradient of the rotation, element by element, on the GPU.

The rotation y = R x of a token is linear, so with respect to x the gradient of <y, w> is R' w, which `inverse` computes. Where x is
one-hot an element of y is one entry of R: a cosine, a sine or its negative, 1 or 0, computed exactly (1 c + 0 s) and rounded once to
bf16. So the entries of both matrices are the same bits, transposed. For any w the gradient's element j is sum_i R_ij w_i, of
one or two terms: within 2^-8 of each term, whose entry R_ij was rounded, 2^-22 of both for fp32 products and sum, and 2^-8 of
the result, which is rounded.
"""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from paged import BF16, cos_sin_table, f64
from test_gpu_cache_moves import axes_of, positions_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

CASES = [  # S, d, rot, begin, inter, axes, how
    (37, 64, 64, 0, False, 3, "cyclic"), (20, 64, 64, 0, True, 1, "none"), (9, 128, 64, 32, False, 2, "random"), (11, 192, 64, 128, True, 3, "sections"),
    (5, 72, 48, 16, False, 1, "none"),
]


def rotations(case):
    """Keywords of the rotation, and its matrices [S, d, d] and those of the way back, from one-hot rows (a head each)."""
    S, d, rot, begin, inter, axes, how = case
    kw = dict(rot_begin=begin, interleaved=inter)
    if how != "none":
        kw.update(positions=positions_of(S, axes, 50).view(1, S, axes).to(DEV), pair_axes=axes_of(rot // 2, axes, how).to(DEV))
    table = cos_sin_table(50, rot).to(DEV)
    x = torch.eye(d, dtype=BF16, device=DEV)[None, :, None].expand(1, d, S, d)
    there, back = (fa.rotate(x, table, inverse=inverse, **kw)[0] for inverse in (False, True))  # [j, s, i]
    return table, kw, there.permute(1, 2, 0), back.permute(1, 2, 0)


def fits(dx, w, matrix):
    """Whether dx [S, d] is the gradient of <R x, w>, R [S, d, d] with rounded entries, in every element."""
    terms = matrix * w[:, :, None]
    want = terms.sum(1)
    bar = (2.0 ** -8 + 2.0 ** -22) * np.abs(terms).sum(1) + 2.0 ** -8 * np.abs(dx)
    return np.all(np.abs(dx - want) <= bar * 1.01)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_the_way_back_is_the_transposed_matrix(case):
    _, _, there, back = rotations(case)
    assert torch.equal(there.transpose(1, 2), back)  # (0 and -0 are equal)
    assert not torch.equal(there, back) and not torch.equal(-there.transpose(1, 2), back)
    assert bool((there != 0).any(2).all())


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients_in_every_element(case):
    S, d, rot, begin, *_ = case
    table, kw, there, _ = rotations(case)
    w = torch.randn(1, 1, S, d, generator=torch.Generator().manual_seed(d)).to(BF16)
    dx, same_way = (f64(fa.rotate(w.to(DEV), table, inverse=inverse, **kw)[0, 0]) for inverse in (True, False))
    matrix, w = f64(there), f64(w)[0, 0]
    assert fits(dx, w, matrix)
    # What would not be the gradient does not pass.
    for wrong in (np.zeros_like(dx), -dx, same_way, w, np.roll(dx, 1, axis=0), dx * (1 + 2.0 ** -5)):
        assert not fits(wrong, w, matrix)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_differences_of_the_loss(case):
    """Steps of 1 along every element of a token, from inputs of small whole numbers (exact): R(x + e) - R(x) is R e within the
    roundings of both, so <w, difference> is the gradient's element within them."""
    S, d, *_ = case
    table, kw, there, _ = rotations(case)
    g = torch.Generator().manual_seed(S)
    x, w = torch.randint(-3, 4, (1, 1, S, d), generator=g).to(BF16), torch.randn(1, 1, S, d, generator=g).to(BF16)
    dx = f64(fa.rotate(w.to(DEV), table, inverse=True, **kw)[0, 0])
    y0 = f64(fa.rotate(x.to(DEV), table, **kw)[0, 0])
    stepped = (x + torch.eye(d, dtype=BF16)[None, :, None]).to(DEV)  # [1, j, s, d]
    y1 = f64(fa.rotate(stepped, table, **kw)[0])
    w64 = f64(w)[0, 0]
    diff = (w64[None] * (y1 - y0[None])).sum(2).T  # [s, j]
    touched = np.abs(f64(there)).transpose(0, 2, 1) > 0  # [s, j, i]: elements of y that x_j reaches; the others cancel exactly
    bar = 2.0 ** -8 * (np.abs(w64)[:, None] * (np.abs(y1.transpose(1, 0, 2)) + np.abs(y0)[:, None]) * touched).sum(2) + 2.0 ** -8 * np.abs(dx)
    off = np.abs(diff - dx)
    assert np.all(off <= bar * 1.01)
    assert (np.abs(diff) > bar).mean() > 0.5 and (np.abs(diff + dx) > bar).mean() > 0.7  # most elements tell a zero, or its negative
