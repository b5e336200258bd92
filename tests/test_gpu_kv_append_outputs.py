"""Where kv_append may write the turned queries: over q, or anywhere that q does not reach."""

import pytest
import torch

import paper_2609_21264_amd as fa

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def call(q, q_out):
    T, hkv, d = q.shape[0], 2, q.shape[2]
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(T, hkv, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    kc, vc = (torch.zeros(2, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    angles = torch.rand(32, d // 2, device="cuda", generator=g)
    return fa.kv_append(k, v, kc, vc, ints([[0, 1]]), ints([20]), ints([0, T]), q=q, q_out=q_out,
                        cos_sin=torch.cat([angles.cos(), angles.sin()], dim=1))


def test_q_and_q_out_in_one_buffer():
    """A program's arena: one allocation that holds both, one behind the other, in either order."""
    T, H, d = 5, 4, 64
    arena = torch.randn(2 * T * H * d + 64, device="cuda").bfloat16()
    n = T * H * d
    for first, second in ((0, n), (n, 0), (0, n + 64)):
        q, q_out = (arena[at:at + n].view(T, H, d) for at in (first, second))
        before = q.clone()
        want = call(q.clone(), None)
        assert call(q, q_out) is q_out
        torch.cuda.synchronize()
        assert torch.equal(q_out, want) and torch.equal(q, before)
    # The halves of a row that begin and end in different tokens' rows: apart as ranges where there is one token.
    row = torch.randn(1, 2 * H, d, device="cuda").bfloat16()
    want = call(row[:, :H].clone(), None)
    call(row[:, :H], row[:, H:])
    torch.cuda.synchronize()
    assert torch.equal(row[:, H:], want)


def test_q_out_that_overlaps_q_is_refused():
    T, H, d = 5, 4, 64
    arena = torch.zeros(4 * T * H * d, dtype=torch.bfloat16, device="cuda")
    n = T * H * d
    q = arena[n:2 * n].view(T, H, d)
    for at in (n - 64, n + 64, n + 8, 2 * n - 8, 8):
        with pytest.raises(ValueError, match="q_out"):
            call(q, arena[at:at + n].view(T, H, d))
    with pytest.raises(ValueError, match="q_out"):  # q's rows in another order
        call(q, arena[n:2 * n].view(H, T, d).transpose(0, 1))
    with pytest.raises(ValueError, match="q_out"):  # ranges that interleave
        call(arena[: 2 * n].view(T, 2 * H, d)[:, :H], arena[: 2 * n].view(T, 2 * H, d)[:, H:])
    call(q, q)
    same = arena[n:2 * n].view(T, H, d)  # q itself, as another tensor
    assert call(q, same) is same
