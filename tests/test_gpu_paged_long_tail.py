"""Attention over a paged cache where one key outweighs each of very many others, which together still count: their
probabilities must not be lost as they are rounded for the product with V."""

import math

import pytest
import torch

import paper_2609_21264_amd as fa

pytestmark = pytest.mark.gpu

PAGE = 1024


def caches(heads, d, dv, fp8, k0, v0, vrest):
    """Two pages: the first key of page 0 has k0 in dim 0 (all other keys are zero) and the value v0, all others vrest."""
    k, v = (torch.zeros(2, heads, PAGE, x, dtype=torch.bfloat16, device="cuda") for x in (d, dv))
    v.fill_(vrest)
    k[0, :, 0, 0], v[0, :, 0] = k0, v0
    return [t.to(torch.float8_e4m3fn) if fp8 else t for t in (k, v)]


# Every workgroup of either kernel takes a whole sequence of one head: 512 items of one row, 256 blocks or more.
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,path", [(512, "few"), (512, "many")])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("below", [22.5, 25.5])
def test_many_small_probabilities(below, d, dv, heads, path, fp8):
    """The first of 2^17 keys has a score `below` powers of two over the others', whose sum is 2^(17 - below). O is 0 for
    the first and 1 for the others, so O = s / (1 + s) with s = (2^17 - 1) 2^-below.

    Bar: P enters the product times 2^7 in fp16 (half a step: 2^-11 of it, at least 2^-25, so 2^-32 unscaled; all in one
    direction, for equal keys) or in bf16 (2^-8 of it); O is rounded once, 2^-8 of it. The fp32 sums take one addition a
    tile of 32 keys and more, 2^12 at most, each off by 2^-24 of the sum: 2^-12 of the row sum (1 to 2) and of O, twice."""
    n, scale = 2 ** 17, below * math.log(2.0)
    kc, vc = caches(heads, d, dv, fp8, 1.0, 0.0, 1.0)
    q = torch.zeros(1, heads, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    table = torch.ones(1, n // PAGE, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    lens, starts = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    o, lse = fa.forward_paged(q, kc, vc, table, lens, starts, max_q=1, scale=scale, return_lse=True, path=path)
    torch.cuda.synchronize()
    s = (n - 1) * 2.0 ** -below
    want = s / (1 + s)
    p_off = n * 2.0 ** -32 + 2.0 ** -11 * want if fp8 else 2.0 ** -8 * want
    bar = p_off + (2.0 ** -8 + 2.0 ** -11) * want
    assert (o.double() - want).abs().max().item() <= bar, (o.min().item(), o.max().item(), want)
    assert (lse.double() - (scale + math.log1p(s))).abs().max().item() <= 2.0 ** -12 + 2.0 ** -20 * (1 + scale)
