"""GPU tests of the attention over a paged cache with many new tokens per sequence (prompts and chunks), against float64."""

import pytest
import torch

import paper_2609_21264_amd as fa
from paged import Batch
from test_gpu_paged import DIMS, run as run_any

pytestmark = pytest.mark.gpu


def run(bt, **kw):
    """The kernel for many rows, whatever the sizes; and what the call chooses by itself."""
    run_any(bt, **kw)
    return run_any(bt, path="many", **kw)


def splits(bt):
    """Whether the kernel for many rows needs a workspace: blocks are split where they would not fill the chip."""
    return fa.fa_fwd_paged_workspace_bytes(len(bt.new), bt.T, bt.table.shape[1] * bt.page, bt.Hq, bt.Hkv, bt.dqk, bt.dv,
                                           fa.FA_CACHE_BF16, max(bt.new), fa.FA_PAGED_MANY) > 0


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("n,extra", [(65, 0), (256, 0), (257, 1), (300, 1000), (100, 5000)])
def test_prompt_and_chunk(n, extra, dqk, dv, page, causal):
    bt = Batch([n], [n + extra], 4, 2, dqk, dv, page, seed=n)
    assert splits(bt)
    run(bt, causal=causal)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (14, 2), (5, 5), (96, 2)])
def test_groups(Hq, Hkv):
    # 256 row-heads of a block end anywhere inside a token's group.
    run(Batch([129, 70], [129, 400], Hq, Hkv, 64, 64, 16, seed=Hq))
    run(Batch([129, 70], [129, 400], Hq, Hkv, 128, 128, 32, seed=Hq + 1))


@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("causal", [True, False])
def test_mixed_lengths(dqk, dv, causal):
    # Single tokens, none, prompts, a chunk, more tokens than keys (a prompt's first rows see nothing).
    run(Batch([1, 300, 0, 5, 131, 1, 200], [1000, 300, 40, 77, 2000, 1, 90], 8, 2, dqk, dv, 16, seed=7), causal=causal)


@pytest.mark.parametrize("dqk,dv,hkv", [(64, 64, 112), (128, 128, 64), (192, 128, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_whole_blocks(dqk, dv, hkv, causal):
    """Enough blocks to fill the chip: none is split."""
    new = [1111, 1111]
    bt = Batch(new, [1111, 1500], hkv, hkv, dqk, dv, 32, seed=3)
    assert not splits(bt)
    run(bt, causal=causal)


def test_whole_blocks_beside_tokens():
    bt = Batch([1, 900, 0, 1, 1033, 2, 77], [300, 900, 9, 5, 1300, 2, 400], 64, 64, 128, 128, 16, seed=5, extra=2)
    run(bt)


@pytest.mark.parametrize("B", [63, 65, 130])
def test_many_sequences(B):
    new = [1 + (37 * i) % 90 for i in range(B)]
    run(Batch(new, [n + (i % 3) * 100 for i, n in enumerate(new)], 4, 2, 64, 64, 16, seed=B))


@pytest.mark.parametrize("causal", [True, False])
def test_pages_that_are_not_there(causal):
    bt = Batch([150, 90, 200], [700, 333, 200], 8, 2, 128, 128, 16, seed=31)
    bt.table[0, 3], bt.table[0, 43] = -1, bt.n_pages
    bt.table[1, 0:4], bt.table[1, 20] = 2 ** 31 - 1, -2 ** 31
    bt.table[2, :] = -1
    bt.d_table = bt.table.cuda()
    run(bt, causal=causal)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 2.0])
def test_scales(scale):
    run(Batch([100, 200], [200, 1500], 4, 2, 64, 64, 16, seed=3), scale=scale)


@pytest.mark.parametrize("dqk,dv", DIMS)
def test_rising_scores_move_the_reference(dqk, dv):
    """Keys that grow along the sequence: the reference maximum of a row is exceeded by far in later tiles, which are
    redone with keys read from their pages."""
    bt = Batch([90, 120], [1500, 120], 4, 2, dqk, dv, 16, seed=11)
    for b, n in enumerate(bt.keys):
        pos = torch.arange(n)
        pages, slots = bt.table[b, pos // 16].long(), pos % 16
        grow = (0.2 + 6.0 * pos / n)[:, None, None]
        bt.k_cache[pages, :, slots] = (bt.k_cache[pages, :, slots].float() * grow).to(torch.bfloat16)
    bt._to("cuda", "hnd")
    run(bt)
    bt.table[0, 40] = -1
    bt.d_table = bt.table.cuda()
    run(bt)


def test_nhd_cache_and_strided_tensors():
    bt = Batch([200, 1, 60], [300, 40, 1027], 8, 2, 128, 128, 16, seed=21, order="nhd")
    qkv = torch.zeros(bt.T, 12, 128, dtype=torch.bfloat16, device="cuda")
    qkv[:, 2:10] = bt.d_q
    bt.d_q = qkv[:, 2:10]
    out = torch.full((8, bt.T, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    run(bt, out=out[:, :, :128].transpose(0, 1))
    assert torch.all(out[:, :, 128:] == 7)


def test_results_do_not_change_between_runs():
    bt = Batch([700, 130, 1], [2000, 130, 500], 8, 2, 128, 128, 16, seed=39)
    first = bt.attend(return_lse=True, path="many")
    for _ in range(3):
        again = bt.attend(return_lse=True, path="many")
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])


def test_prompt_equals_fused_forward():
    """A prompt without a cached part through its pages and through forward(): the same to rounding."""
    bt = Batch([1000], [1000], 8, 2, 128, 128, 16, seed=51)
    o, lse = run(bt)
    pos = torch.arange(1000)
    k, v = (c[bt.table[0, pos // 16].long(), :, pos % 16].transpose(0, 1)[None].contiguous().cuda()
            for c in (bt.k_cache, bt.v_cache))
    ro, rl = fa.forward(bt.d_q.transpose(0, 1)[None].contiguous(), k, v, causal=True, return_lse=True)
    # Both round P and O to bf16: 2 (2^-8 + 2^-8) max|V|.
    assert (o.float() - ro[0].transpose(0, 1).float()).abs().max() <= 2.0 ** -6 * v.float().abs().max()
    assert (lse - rl[0].T).abs().max() <= 1e-4


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("n,extra,page", [(65, 0, 16), (257, 1, 64), (300, 1000, 32), (100, 5000, 16)])
def test_prompt_and_chunk_e4m3(n, extra, page, dqk, dv, causal):
    run(Batch([n], [n + extra], 4, 2, dqk, dv, page, True, seed=n), causal=causal)


@pytest.mark.parametrize("dqk,dv", DIMS)
def test_mixed_lengths_e4m3(dqk, dv):
    run(Batch([1, 300, 0, 5, 131, 1, 200], [1000, 300, 40, 77, 2000, 1, 90], 8, 2, dqk, dv, 16, True, seed=7))
    bt = Batch([150, 90, 200], [700, 333, 200], 14, 2, dqk, dv, 16, True, seed=31)
    bt.table[0, 3], bt.table[0, 43] = -1, bt.n_pages
    bt.table[1, 0:4], bt.table[1, 20] = 2 ** 31 - 1, -2 ** 31
    bt.table[2, :] = -1
    bt.d_table = bt.table.cuda()
    run(bt)


def test_whole_blocks_e4m3():
    bt = Batch([1111, 1111], [1111, 1500], 64, 64, 128, 128, 32, True, seed=3)
    run(bt)


@pytest.mark.parametrize("ks", [0.0, -0.02, 1e-42])
def test_e4m3_scales(ks):
    """Scales that are zero, negative or tiny (masked scores stay masked), in both kernels."""
    for n in (1, 90):
        bt = Batch([n, n], [n, 300], 4, 2, 128, 128, 16, True, seed=61)
        bt.k_scale = torch.tensor([ks, 0.01])
        bt.d_k_scale = bt.k_scale.cuda()
        run(bt)


@pytest.mark.parametrize("dqk,dv", DIMS)
def test_rising_scores_move_the_reference_e4m3(dqk, dv):
    bt = Batch([90, 120], [1500, 120], 4, 2, dqk, dv, 16, True, seed=11)
    for b, n in enumerate(bt.keys):
        pos = torch.arange(n)
        pages, slots = bt.table[b, pos // 16].long(), pos % 16
        grow = (0.1 + 2.0 * pos / n)[:, None, None]
        rows = (bt.k_cache.float()[pages, :, slots] * grow).clamp(-448, 448).to(bt.k_cache.dtype)
        bt.k_cache.view(torch.uint8)[pages, :, slots] = rows.view(torch.uint8)
    bt._to("cuda", "hnd")
    run(bt)
    bt.table[0, 40] = -1
    bt.d_table = bt.table.cuda()
    run(bt)


@pytest.mark.parametrize("dqk,dv", DIMS[:2])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [17, 31, 32])
def test_short_blocks(n, dqk, dv, causal):
    """Up to 128 row-heads per key/value head: blocks of 128, split, beside other lengths and whole."""
    run(Batch([n], [4000], 8, 2, dqk, dv, 16, seed=n), causal=causal)
    run(Batch([n, 1, 0, n], [n, 700, 30, 1501], 8, 2, dqk, dv, 64, seed=n), causal=causal)
    bt = Batch([n] * 20, [n + 37 * i for i in range(20)], 256, 64, dqk, dv, 16, seed=n)
    assert not splits(bt)
    run(bt, causal=causal)


def test_short_blocks_page_windows_and_holes():
    bt = Batch([32], [70 * 64], 4, 1, 128, 128, 16, seed=71)  # more tiles than a register of page numbers holds
    run(bt)
    bt.table[0, 0:8] = -1
    bt.table[0, 200], bt.table[0, -1] = bt.n_pages, -1
    bt.d_table = bt.table.cuda()
    run(bt)


@pytest.mark.parametrize("path", [None, "few", "many"])
@pytest.mark.parametrize("dqk,dv,Hq,Hkv", [(64, 64, 128, 16), (128, 128, 64, 8), (192, 128, 64, 32)])
def test_paths_by_work(path, dqk, dv, Hq, Hkv):
    """Batches around the work from which prompts go to the kernel for many rows, beside single tokens (by themselves the
    two kernels share the sequences then), and a table wider than its lengths."""
    for keys in (400, 2100):
        bt = Batch([230, 1, 0, 9, 120], [keys, 500, 3, 80, 333], Hq, Hkv, dqk, dv, 32, seed=keys, blocks=100)
        run_any(bt, path=path)


def test_paths_many_sequences():
    new = [1 + (31 * i) % 60 for i in range(150)]
    run_any(Batch(new, [n + 10 * (i % 50) for i, n in enumerate(new)], 64, 4, 64, 64, 16, seed=77, blocks=60))


@pytest.mark.parametrize("keys", [[2000, 1], [300, 300], [64, 2048]])
def test_captured_call_serves_short_and_long_prompts(keys):
    """Which kernel takes the prompts is decided on the device, so a captured call serves both."""
    bt = Batch([150, 150], [2048, 2048], 64, 8, 128, 128, 16, seed=79)
    T = bt.T
    out, lse = torch.empty(T, 64, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 64, device="cuda")
    bt.attend(out=out, lse=lse, return_lse=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bt.attend(out=out, lse=lse, return_lse=True)
    for lens in ([2048, 2048], keys, [2048, 150], keys):
        bt.kv_lens = torch.tensor(lens, dtype=torch.int32)
        bt.d_kv_lens.copy_(bt.kv_lens)
        out.fill_(float("nan"))
        graph.replay()
        bt.check(out, lse, 128 ** -0.5, True, str(lens))
