"""GPU tests of the attention over a paged cache by probability mass (paged_mass.py): bars relative to every output element,
so that a lost or doubled tile, a part's wrong weight or a misread value shows however many keys there are."""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle.paged import rotate
from paged import E4M3, cos_sin_table, f64
from paged_mass import KINDS, check_mass, classes, mass_batch

pytestmark = pytest.mark.gpu

DIMS = [(64, 64), (128, 128), (192, 128)]


def run(bt, causal=True, scale=None, **kw):
    scale = bt.dqk ** -0.5 if scale is None else scale
    o, lse = bt.attend(causal=causal, scale=scale, return_lse=True, **kw)
    torch.cuda.synchronize()
    check_mass(bt, o, scale, causal)
    return o, lse


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_one_token_over_many_parts(dqk, dv, fp8, kind):
    run(mass_batch(kind, [1], [9001], 4, 1, dqk, dv, 16, fp8, seed=1))
    run(mass_batch(kind, [1, 2], [5003, 2049], 3, 3, dqk, dv, 64, fp8, seed=2, order="nhd"))
    run(mass_batch(kind, [1, 1, 1, 1], [1, 129, 640, 3000], 8, 2, dqk, dv, 32, fp8, seed=3))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (64, 1), (4, 1), (16, 16)])
def test_joins(Hq, Hkv, fp8):
    """Items of up to hundreds of parts, with few columns and with many."""
    for kind in KINDS:
        run(mass_batch(kind, [1], [40000], Hq, Hkv, 128, 128, 64, fp8, seed=Hq))


@pytest.mark.parametrize("path", ["few", "many", None])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_draft_tokens_prompts_and_chunks(dqk, dv, fp8, path):
    for causal in (True, False):
        run(mass_batch("blocks", [5, 9, 17], [3001, 700, 90], 8, 2, dqk, dv, 16, fp8, seed=5), causal, path=path)
        run(mass_batch("residues", [70, 1, 130], [1500, 900, 130], 4, 2, dqk, dv, 32, fp8, seed=6), causal, path=path)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dqk,dv", DIMS)
def test_blocks_that_are_split(dqk, dv, fp8, kind):
    # 300 tokens of two heads over many keys: each block in several parts; and one beside single tokens.
    run(mass_batch(kind, [300], [5000], 4, 2, dqk, dv, 16, fp8, seed=7), path="many")
    run(mass_batch(kind, [1, 200, 1], [2500, 4003, 800], 4, 1, dqk, dv, 64, fp8, seed=8))


@pytest.mark.parametrize("dqk,dv,heads", [(64, 64, 112), (128, 128, 64), (192, 128, 64)])
@pytest.mark.parametrize("fp8", [False, True])
def test_whole_blocks(dqk, dv, heads, fp8):
    run(mass_batch("blocks", [555, 600], [555, 900], heads, heads, dqk, dv, 32, fp8, seed=9), path="many")


@pytest.mark.parametrize("path", ["few", "many"])
def test_pages_that_are_not_there(path):
    bt = mass_batch("blocks", [1, 40], [9000, 1500], 4, 2, 128, 128, 16, seed=11)
    bt.table[0, 100:140], bt.table[0, 562], bt.table[1, 0], bt.table[1, 60] = -1, bt.n_pages, -5, 2 ** 31 - 1
    bt.d_table = bt.table.cuda()
    run(bt, path=path)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("path", ["few", "many"])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30, 0.5])
def test_scales(scale, path, fp8):
    run(mass_batch("residues", [1, 50, 3], [5000, 700, 90], 8, 2, 128, 128, 16, fp8, seed=12), scale=scale, path=path)


@pytest.mark.parametrize("path", ["few", "many"])
def test_requests_that_share_their_pages(path):
    """One table row for all requests (a row stride of 0), each with its own length: the sequences of a shared prompt."""
    one = mass_batch("blocks", [0], [3000], 8, 2, 128, 128, 16, seed=15)
    lens = [3000, 1, 17, 2999, 640]
    bt = mass_batch("blocks", [1, 1, 9, 30, 1], lens, 8, 2, 128, 128, 16, seed=16)  # for its queries and starts
    table = one.d_table.expand(len(lens), -1)
    o = fa.forward_paged(bt.d_q, one.d_k_cache, one.d_v_cache, table, bt.d_kv_lens, bt.d_q_starts, path=path)
    own = fa.forward_paged(bt.d_q, one.d_k_cache, one.d_v_cache, table.contiguous(), bt.d_kv_lens, bt.d_q_starts, path=path)
    assert table.stride(0) == 0 and torch.equal(o, own)
    for b, n in enumerate(lens):  # each against the check, as a batch of its own (classes by its own length: as all 3 000 keys have)
        q0, q1 = int(bt.q_starts[b]), int(bt.q_starts[b + 1])
        alone = fa.forward_paged(bt.d_q[q0:q1], one.d_k_cache, one.d_v_cache, one.d_table, bt.d_kv_lens[b:b + 1],
                                 torch.tensor([0, q1 - q0], dtype=torch.int32, device="cuda"), path=path)
        # Cut elsewhere and joined: P and O rounded twice, in each run.
        assert (o[q0:q1].double() - alone.double()).abs().le(2 * (2.0 ** -8 + 2.0 ** -8 + 1e-3) * alone.double() + 1e-6).all(), n


@pytest.mark.parametrize("dqk,dv,page,fp8", [(128, 128, 16, False), (64, 64, 32, True), (192, 128, 64, False)])
def test_serving_run(dqk, dv, page, fp8):
    """Append and attend, a ragged prompt, a second chunk beside single tokens, then single tokens. The values appended are the
    one-hot rows of their positions, so every step's output tells which positions it saw with which weight; keys are
    checked against the rotated inputs, by one rounding."""
    Hq, Hkv, steps = 8, 2, [[100, 17, 1], [150, 1, 1], [1, 1, 1], [1, 0, 1], [1, 1, 3]]
    final = np.sum(steps, axis=0).tolist()
    bt = mass_batch("residues", [0, 0, 0], final, Hq, Hkv, dqk, dv, page, fp8, seed=13)
    if fp8:  # an appended 1.0 becomes 1 / scale: an exact power of two
        bt.v_scale = torch.full((Hkv,), 2.0 ** -6)
        bt.d_v_scale = bt.v_scale.cuda()
    table = cos_sin_table(bt.table.shape[1] * page, dqk)
    raw = torch.uint8 if fp8 else torch.int16
    for c in (bt.d_k_cache, bt.d_v_cache):
        c.view(raw).fill_(0x7F if fp8 else 0x7FC0)  # nothing but NaN at the start
    g = torch.Generator().manual_seed(14)
    held, seen, d_table = np.zeros(3, dtype=np.int64), [[], [], []], table.cuda()
    for n in steps:
        held += n
        T = sum(n)
        q, k = (torch.randn(T, h, dqk, generator=g).bfloat16().cuda() for h in (Hq, Hkv))
        pos = np.concatenate([np.arange(held[b] - n[b], held[b]) for b in range(3)])
        v = torch.zeros(T, Hkv, dv)
        v[torch.arange(T), :, torch.from_numpy(classes("residues", 1 << 20, dv)[pos])] = 1.0
        bt.q_starts = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32)
        bt.kv_lens, bt.keys, bt.new, bt.T = torch.tensor(held, dtype=torch.int32), held.tolist(), n, T
        args = (bt.d_k_cache, bt.d_v_cache, bt.d_table, bt.kv_lens.cuda(), bt.q_starts.cuda())
        scales = {"k_scale": bt.d_k_scale, "v_scale": bt.d_v_scale}
        qr = fa.kv_append(k, v.bfloat16().cuda(), *args, q=q, cos_sin=d_table, **scales)
        o = fa.forward_paged(qr, *args, max_q=max(n), **scales)
        torch.cuda.synchronize()
        bt.q, bt.k_cache = qr.cpu(), bt.d_k_cache.cpu()
        if fp8:  # the oracle's value is one_hot * v_scale of stored ones; here one_hot itself was appended
            check_mass(bt, f64(o) * 2.0 ** -6, dqk ** -0.5, True, str(n))
        else:
            check_mass(bt, o, dqk ** -0.5, True, str(n))
        tab = table.double().numpy()
        for b in range(3):
            for i in range(n[b]):
                p = int(held[b]) - n[b] + i
                seen[b].append(rotate(f64(k[int(bt.q_starts[b]) + i]), tab[p, : dqk // 2], tab[p, dqk // 2:], 0, False))
    kc, vc = bt.values(bt.d_k_cache, bt.k_scale), bt.values(bt.d_v_cache, bt.v_scale)
    for b in range(3):
        want, pos = np.stack(seen[b]), np.arange(final[b])
        rows = bt.table[b, pos // page].numpy()
        sc = f64(bt.k_scale)[:, None] if fp8 else 1.0
        step = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * sc) if fp8 else 2.0 ** -8 * np.abs(want)
        assert np.all(np.abs(kc[rows, :, pos % page] - want) <= step + 2.0 ** -20 * np.abs(want).max())
        hot = np.zeros((final[b], dv))
        hot[pos, classes("residues", final[b], dv)] = 1.0
        assert np.array_equal(vc[rows, :, pos % page], np.repeat(hot[:, None], Hkv, axis=1))
    assert (bt.d_v_cache.dtype == E4M3) == fp8


def test_appends_past_32_bits_land_where_they_belong():
    """A cache of 4.5 GiB a buffer: all appended keys and values lie in its last pages, bit for bit, and neither the places
    whose offsets are 2^32 bytes lower nor any other changed."""
    pages, page, heads, d = 73728, 64, 4, 128
    assert pages * page * heads * d * 2 > 2 ** 32
    kc = torch.zeros(pages, heads, page, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    table = torch.tensor([[pages - 1, pages - 3], [pages - 2, -1]], dtype=torch.int32, device="cuda")
    lens, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([100, 64], [0, 40, 42]))
    k, v = (torch.randn(42, heads, d, device="cuda").bfloat16() for _ in range(2))
    fa.kv_append(k, v, kc, vc, table, lens, starts)
    torch.cuda.synchronize()
    for x, c in ((k, kc), (v, vc)):
        want = torch.zeros(3, heads, page, d, dtype=torch.bfloat16, device="cuda")  # pages -3, -2, -1
        want[2, :, 60:64], want[0, :, 0:36] = x[:4].transpose(0, 1), x[4:40].transpose(0, 1)
        want[1, :, 62:64] = x[40:].transpose(0, 1)
        assert torch.equal(c[-3:], want)
        assert not any(part.any() for part in c[:-3].split(8192))
