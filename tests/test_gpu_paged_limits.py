"""GPU tests of the paged calls at sizes where a grid or a count passes a limit."""

import pytest
import torch

import paper_2609_21264_amd as fa
from paged import Batch

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("T", [2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, 2 ** 24 + 5])
def test_append_of_very_many_tokens(T):
    """2^24 workgroups of 256 threads are more than one dimension of a grid holds. Two sequences: nearly all tokens, and
    the last three."""
    g = torch.Generator(device="cuda").manual_seed(T)
    page, split = 64, T - 3
    # Rows 8 elements apart, so that every token has its own and the buffers stay small.
    k, v, q = (torch.randn(8 * (T + 8), device="cuda", generator=g).bfloat16().as_strided((T, 1, 64), (8, 8, 1)) for _ in range(3))
    blocks = -(-split // page)
    kc, vc = (torch.zeros(blocks + 1, 1, page, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.zeros(2, blocks, dtype=torch.int32, device="cuda")
    table[0] = torch.arange(blocks, dtype=torch.int32, device="cuda")
    table[1, 0] = blocks
    q_out = torch.zeros(T, 1, 64, dtype=torch.bfloat16, device="cuda")
    fa.kv_append(k, v, kc, vc, table, ints([split, 3]), ints([0, split, T]), q=q, q_out=q_out)
    torch.cuda.synchronize()
    for x, cache in ((k, kc), (v, vc)):
        rows = cache.view(-1, 64)
        assert torch.equal(rows[:split], x[:split, 0]), "the first sequence"
        assert torch.equal(rows[blocks * page:blocks * page + 3], x[split:, 0]), "the second"
        assert not rows[split:blocks * page].any() and not rows[blocks * page + 3:].any()
    assert torch.equal(q_out, q)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,keys,Hq,Hkv", [([1024] + [1] * 24, [3000] + [700] * 24, 8, 2), ([1] * 40 + [600], [90] * 41, 4, 2),
                                             ([1] * 33, [40 * i + 1 for i in range(33)], 8, 2), ([0, 0, 3], [5, 0, 900], 8, 2),
                                             ([300, 280, 290], [300, 280, 1290], 4, 4)], ids=str)
def test_without_max_q(new, keys, Hq, Hkv, fp8):
    """The call as most programs write it first: no hint at all."""
    keys = [max(n, k) for n, k in zip(new, keys)]
    bt = Batch(new, keys, Hq, Hkv, 128, 128, 16, fp8, seed=len(new))
    for causal in (True, False):
        o, lse = bt.attend(max_q=None, causal=causal, return_lse=True)
        bt.check(o, lse, 128 ** -0.5, causal, str(new[:3]))


@pytest.mark.parametrize("keys", [300, 6000])
@pytest.mark.parametrize("path", ["few", "many", None])
def test_starts_that_decrease_stay_inside_the_buffers(path, keys):
    """Results are undefined where q_starts decreases; what lies around the outputs and the workspace is not touched, and the
    next call is right."""
    bt = Batch([40, 1, 60, 3], [keys] * 4, 8, 2, 128, 128, 16, seed=keys)
    want = bt.attend(return_lse=True, path=path)
    o, lse = (torch.full((bt.T + 2, 8, *x), 7.0, dtype=t, device="cuda") for x, t in (((128,), torch.bfloat16), ((), torch.float32)))
    n = fa.fa_fwd_paged_workspace_bytes(4, bt.T, bt.table.shape[1] * 16, 8, 2, 128, 128, 0, 60,
                                        {"few": 1, "many": 2, None: 0}[path])
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    right = bt.d_q_starts.clone()
    for starts in ([0, bt.T, 0, bt.T, 0], [bt.T, 0, bt.T, 50, 60], [-5, 2 ** 31 - 1, -2 ** 31, 70, 30]):
        bt.d_q_starts.copy_(ints(starts))
        bt.attend(out=o[1:-1], lse=lse[1:-1], workspace=ws[:n], path=path, return_lse=True)
        torch.cuda.synchronize()
        assert all((t[i] == 7).all() for t in (o, lse) for i in (0, -1)) and (ws[n:] == 0x5A).all()
    bt.d_q_starts.copy_(right)
    again = bt.attend(return_lse=True, path=path)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
