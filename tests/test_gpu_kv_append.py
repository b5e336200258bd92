"""GPU tests of appending to a paged cache with the position rotation (fa_kv_append), against float64, and of a serving
run of append and attention together."""

import numpy as np
import pytest
import torch

import paper_2609_21264_amd as fa
from oracle import attention_head
from oracle.paged import rotate, token_positions
from paged import BF16, E4M3, Batch, cos_sin_table, f64

pytestmark = pytest.mark.gpu

# (dqk, dv, rotated dims, first, neighbouring pairs)
ROTATIONS = [(64, 64, 64, 0, False), (128, 128, 128, 0, False), (128, 128, 128, 0, True), (128, 128, 32, 0, False),
             (128, 128, 48, 40, False), (128, 128, 8, 120, True), (192, 128, 64, 128, True), (192, 128, 192, 0, False),
             (192, 128, 0, 0, False), (64, 64, 16, 8, True)]


def expected(bt, x, table, begin, inter, pos):
    """Token rows in float64 after the rotation, and the sum of the magnitudes in each element's pair."""
    x = f64(x)
    y, mag = x.copy(), np.abs(x)
    if table is not None:
        tab = table.double().numpy()
        half = tab.shape[1] // 2
        for t, (b, p) in enumerate(pos):
            if b >= 0:
                y[t] = rotate(x[t], tab[p, :half], tab[p, half:], begin, inter)
                for sign in (1.0, -1.0):  # |x| + |y| comes out at one element of the pair for each sign
                    mag[t] = np.maximum(mag[t], np.abs(rotate(np.abs(x[t]), np.ones(half), sign * np.ones(half), begin, inter)))
    return y, mag


def check_append(bt, table, begin, inter, q_out):
    torch.cuda.synchronize()
    pos = token_positions(bt.q_starts, bt.kv_lens)
    rows = [t for t, (b, _) in enumerate(pos) if b >= 0]
    if q_out is not None:
        y, mag = expected(bt, bt.q, table, begin, inter, pos)
        off = np.abs(f64(q_out)[rows] - y[rows]) - (2.0 ** -8 * np.abs(y[rows]) + 2.0 ** -21 * mag[rows])
        assert off.max(initial=-1) <= 0
    for name, x, cache, d_cache, scale, tab in (("k", bt.k, bt.k_cache, bt.d_k_cache, bt.k_scale, table),
                                                ("v", bt.v, bt.v_cache, bt.d_v_cache, bt.v_scale, None)):
        y, mag = expected(bt, x, tab, begin, inter, pos)
        raw = torch.uint8 if bt.fp8 else torch.int16
        before, after = cache.view(raw).numpy().copy(), d_cache.contiguous().view(raw).cpu().numpy()
        got = f64(d_cache)
        for t in rows:
            b, p = pos[t]
            pg, slot = int(bt.table[b, p // bt.page]), p % bt.page
            if not 0 <= pg < bt.n_pages:
                continue
            if bt.fp8:
                sc = f64(scale)[:, None]
                want, m = np.clip(y[t] / sc, -448, 448), mag[t] / sc
                bar = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + 2.0 ** -20 * m
            else:
                want, bar = y[t], 2.0 ** -8 * np.abs(y[t]) + 2.0 ** -21 * mag[t]
            off = np.abs(got[pg, :, slot] - want) - bar
            assert off.max() <= 0, (name, t, b, p)
            before[pg, :, slot] = after[pg, :, slot]
            if tab is None and not bt.fp8:  # copied as it is
                assert np.array_equal(got[pg, :, slot], f64(x)[t])
        assert np.array_equal(before, after), f"{name}: something else was written"


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rot", ROTATIONS, ids=str)
def test_append(rot, fp8):
    dqk, dv, n, begin, inter = rot
    # ragged, without a token, more tokens than keys (those before position 0 are left out)
    bt = Batch([1, 7, 0, 33, 5, 2], [300, 7, 20, 50, 3, 64], 6, 3, dqk, dv, 16, fp8, seed=n + begin, extra=3)
    table = cos_sin_table(bt.table.shape[1] * 16, n) if n else None
    q_out = torch.full_like(bt.d_q, 9.0)
    r = bt.append(q=bt.d_q, q_out=q_out, cos_sin=None if table is None else table.cuda(), rot_begin=begin, interleaved=inter)
    assert r is q_out
    check_append(bt, table, begin, inter, q_out)
    pos = token_positions(bt.q_starts, bt.kv_lens)
    left = [t for t, (b, _) in enumerate(pos) if b < 0] + list(range(len(pos), bt.T))
    assert len(left) == 5 and torch.all(q_out[left] == 9)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (32, 8), (71, 71), (0, 2)])
def test_append_heads(Hq, Hkv):
    bt = Batch([1, 3], [17, 90], max(Hq, Hkv), Hkv, 128, 128, 32, seed=Hq)
    table = cos_sin_table(bt.table.shape[1] * 32, 128)
    q = bt.append(q=bt.d_q if Hq else None, cos_sin=table.cuda())
    check_append(bt, table, 0, False, q)


@pytest.mark.parametrize("B", [62, 63, 64, 65, 4095, 5000])
def test_append_many_sequences(B):
    # The search for a token's sequence takes 64 probes at a time: one step up to 63 sequences, two up to 4 095.
    new = np.random.RandomState(B).choice([0, 0, 1, 2], B).tolist()
    bt = Batch(new, [n + i % 5 for i, n in enumerate(new)], 1, 1, 64, 64, 16, seed=B, extra=2)
    check_append(bt, None, 0, False, bt.append(q=bt.d_q))


@pytest.mark.parametrize("fp8", [False, True])
def test_append_in_place_from_a_fused_buffer(fp8):
    bt = Batch([3, 2], [40, 18], 8, 2, 128, 128, 16, fp8, seed=3, order="nhd")
    table = cos_sin_table(bt.table.shape[1] * 16, 64)
    qkv = torch.cat([bt.d_q, bt.d_k, bt.d_v], dim=1)
    q, bt.d_k, bt.d_v = qkv.split([8, 2, 2], dim=1)
    r = bt.append(q=q, q_out=q, cos_sin=table.cuda())
    assert r.data_ptr() == qkv.data_ptr()
    check_append(bt, table, 0, False, q)
    assert torch.equal(qkv[:, 8:10].cpu(), bt.k) and torch.equal(qkv[:, 10:].cpu(), bt.v)


def test_append_to_pages_that_are_not_there():
    bt = Batch([4, 3], [20, 40], 2, 2, 64, 64, 16, seed=5)
    bt.table[0, 1], bt.table[1, 2] = bt.n_pages, -1
    bt.d_table = bt.table.cuda()
    table = cos_sin_table(bt.table.shape[1] * 16, 64)
    check_append(bt, table, 0, False, bt.append(q=bt.d_q, cos_sin=table.cuda()))


def test_append_e4m3_extremes():
    """What passes the largest value becomes it, infinities too; NaN stays NaN; small values round to nearest even."""
    bt = Batch([1], [1], 1, 1, 64, 64, 16, True, seed=7)
    ones = torch.ones(1, device="cuda")
    v = torch.zeros(1, 1, 64)
    vals = [448.0, 449.0, 464.0, 480.0, 1e30, float("inf"), -float("inf"), float("nan"), 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10,
            -(2.0 ** -10), 17.0, 18.0, 19.0, 0.0]
    v[0, 0, : len(vals)] = torch.tensor(vals)
    bt.d_v = v.to(BF16).cuda()
    bt.d_k_scale = bt.d_v_scale = ones
    bt.append()
    got = bt.d_v_cache[int(bt.table[0, 0]), 0, 0].float().cpu()[: len(vals)].tolist()
    want = [448.0, 448.0, 448.0, 448.0, 448.0, 448.0, -448.0, None, 2.0 ** -9, 0.0, 2.0 ** -8, -0.0, 16.0, 18.0, 20.0, 0.0]
    assert got[7] != got[7]
    assert [x for i, x in enumerate(got) if i != 7] == [x for i, x in enumerate(want) if i != 7]


def test_append_captured():
    bt = Batch([1, 1], [33, 64], 4, 2, 128, 128, 16, seed=9)
    table = cos_sin_table(bt.table.shape[1] * 16, 128)
    d_table, q_out = table.cuda(), torch.empty_like(bt.d_q)
    bt.append(q=bt.d_q, q_out=q_out, cos_sin=d_table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bt.append(q=bt.d_q, q_out=q_out, cos_sin=d_table)
    for keys in ([33, 64], [1, 20], [16, 17]):
        bt.kv_lens = torch.tensor(keys, dtype=torch.int32)
        bt.d_kv_lens.copy_(bt.kv_lens)
        for name in ("k_cache", "v_cache"):
            getattr(bt, "d_" + name).copy_(getattr(bt, name))
        graph.replay()
        check_append(bt, table, 0, False, q_out)


@pytest.mark.parametrize("dqk,dv,page,fp8", [(128, 128, 16, False), (64, 64, 32, True), (192, 128, 64, False)])
def test_serving_run(dqk, dv, page, fp8):
    """Three requests: ragged prompts, then a second chunk of one beside single tokens, then steps of single tokens; each
    call appends and attends. Checked against float64 attention over the keys and values that the cache holds, and what
    it holds against the rotated inputs."""
    Hq, Hkv, steps = 8, 2, [[100, 17, 1], [150, 1, 1], [1, 1, 1], [1, 0, 1], [1, 1, 3]]
    final = np.sum(steps, axis=0)
    whole = Batch([0, 0, 0], final.tolist(), Hq, Hkv, dqk, dv, page, fp8, seed=11)
    table = cos_sin_table(whole.table.shape[1] * page, dqk)
    d_table = table.cuda()
    held = np.zeros(3, dtype=np.int64)
    raw = torch.uint8 if fp8 else torch.int16
    for c in (whole.d_k_cache, whole.d_v_cache):
        c.view(raw).fill_(0x7F if fp8 else 0x7FC0)  # nothing but NaN at the start
    g = torch.Generator().manual_seed(12)
    seen = [[], [], []]  # appended keys of every request, in float64
    for n in steps:
        held += n
        T = sum(n)
        q, k, v = (torch.randn(T, h, d, generator=g).to(BF16).cuda() for h, d in ((Hq, dqk), (Hkv, dqk), (Hkv, dv)))
        starts = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda")
        lens = torch.tensor(held, dtype=torch.int32, device="cuda")
        args = (whole.d_k_cache, whole.d_v_cache, whole.d_table, lens, starts)
        scales = {"k_scale": whole.d_k_scale, "v_scale": whole.d_v_scale}
        qr = fa.kv_append(k, v, *args, q=q, cos_sin=d_table, **scales)
        o, lse = fa.forward_paged(qr, *args, max_q=max(n), return_lse=True, **scales)
        torch.cuda.synchronize()
        step = Batch.__new__(Batch)
        step.__dict__.update(whole.__dict__)
        step.q, step.kv_lens, step.q_starts = qr.cpu(), lens.cpu(), starts.cpu()
        step.k_cache, step.v_cache = whole.d_k_cache.cpu(), whole.d_v_cache.cpu()
        step.check(o, lse, dqk ** -0.5, True, str(n))
        tab = table.double().numpy()
        for b in range(3):
            for i in range(n[b]):
                p = int(held[b]) - n[b] + i
                seen[b].append(rotate(f64(k[int(starts[b]) + i]), tab[p, : dqk // 2], tab[p, dqk // 2:], 0, False))
    kc = whole.values(whole.d_k_cache, whole.k_scale)
    for b in range(3):
        want = np.stack(seen[b])
        pos = np.arange(len(want))
        got = kc[whole.table[b, pos // page].numpy(), :, pos % page]
        step = 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * 0.02 if fp8 else 2.0 ** -8 * np.abs(want)
        assert np.all(np.abs(got - want) <= step + 2.0 ** -20 * np.abs(want).max())
    # The last row of the longest request once more, from the inputs' keys alone.
    o_ref, _ = attention_head(f64(qr[0, :1]), np.stack(seen[0])[:, 0],
                              whole.values(whole.d_v_cache, whole.v_scale)[whole.table[0, np.arange(final[0]) // page].numpy(), 0,
                                                                           np.arange(final[0]) % page], dqk ** -0.5, True)
    # Keys off by half a step h = 2^-8 (2^-4) relative move a score by at most h |q| |k| scale, so O by at most
    # (exp(2 delta) - 1) max|V| beside the roundings of the call.
    delta = (2.0 ** -4 if fp8 else 2.0 ** -8) * np.abs(f64(qr[0, 0])).sum() * np.abs(np.stack(seen[0])).max() * dqk ** -0.5
    vmax = 6.0
    assert np.abs(f64(o[0, 0]) - o_ref[0]).max() <= (np.expm1(2 * delta) + 2.0 ** -7 + 1e-5) * vmax
