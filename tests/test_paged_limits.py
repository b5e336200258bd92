"""Sizes at the borders of what the paged calls count and launch, on the host (no GPU needed)."""

import pytest

import paper_2609_21264_amd as fa

MANY = fa.FA_PAGED_MANY


def workspace(B, T, keys, Hq, Hkv, d=128, type=0, max_q=1, path=MANY):
    return fa.fa_fwd_paged_workspace_bytes(B, T, keys, Hq, Hkv, d, d, type, max_q, path)


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_split_blocks_lie_on_a_line_that_32_bits_count(d, type):
    """The kernel for many rows splits blocks (and needs a workspace) only where all of them, 4 units and one per 64
    keys each, are fewer than 2^31 units: what lay behind would not be run."""
    assert workspace(248, 248, 2 ** 30, 1, 1, d, type) == 0      # 248 sequences of one token and 2^30 keys: 4.2e9 units
    assert workspace(100, 100, 2 ** 30, 1, 1, d, type) > 0       # 1.7e9
    for blocks in (1, 7, 100, 127, 128, 129, 200, 250):
        for keys in (2 ** 20, 2 ** 28, 2 ** 29, 2 ** 30 - 2 ** 20, 2 ** 30):
            units = 4 + -(-keys // 64)
            split = workspace(blocks, blocks, keys, 1, 1, d, type) > 0
            assert split or (blocks + blocks // 128) * units >= 2 ** 31, (blocks, keys)  # what the host takes for the most
            assert not split or blocks * units < 2 ** 31, (blocks, keys)


def test_a_negative_page_size_is_refused():
    """Before any product or quotient is formed from it: max_blocks * page_size / 128 + 2 is 0 for -256."""
    import test_paged_host as host

    for page in (-1, -16, -255, -256, -383, -2 ** 31):
        for blocks in (0, 1, 4):
            bt = host.batch(max_blocks=blocks)
            assert host.attend(host.cache(page_size=page), bt) == fa.FA_ERR_BAD_SHAPE, page
            assert host.append(host.cache(page_size=page), bt) == fa.FA_ERR_BAD_SHAPE, page


def test_more_blocks_than_a_grid_holds():
    """The kernel for many rows launches up to (T * group / 128 + sequences with rows) * Hkv workgroups of 256 threads,
    fewer than 2^24: the path refuses more, and without a path such a call runs in the kernel for few rows."""
    import test_paged_host as host

    heads = dict(Hkv=8, k_page=8 * 16 * 128, v_page=8 * 16 * 128)
    many = host.batch(B=2 ** 21, T=2 ** 21, max_blocks=1, table_stride=1)
    assert host.attend(host.cache(**heads), many, Hq=8, path=MANY) == fa.FA_ERR_BAD_SHAPE
    fewer = host.batch(B=2 ** 21 - 2 ** 14, T=2 ** 21 - 2 ** 14, max_blocks=1, table_stride=1)
    assert host.attend(host.cache(**heads), fewer, Hq=8, path=MANY, Q=None) == fa.FA_ERR_NULL_POINTER  # sizes are right
    # Sequences of 65 and more row-heads alone, if max_q is right: the kernel for many rows needs no workspace, that for few does.
    n, keys = 2 ** 21, 1024
    few, auto = (workspace(n, 9 * n, keys, 64, 8, max_q=9, path=x) for x in (fa.FA_PAGED_FEW, fa.FA_PAGED_AUTO))
    assert auto == few > 0
    assert workspace(n // 2, 9 * (n // 2), keys, 64, 8, max_q=9, path=fa.FA_PAGED_AUTO) == 0


@pytest.mark.parametrize("new,Hq,Hkv", [((1024,) + (1,) * 24, 32, 8), ((4096,) + (1,) * 255, 16, 8), ((700, 0, 0, 2), 8, 8)], ids=("a", "b", "c"))
@pytest.mark.parametrize("type", [0, 1])
def test_without_max_q_both_kernels_are_launched_for_a_mix(new, Hq, Hkv, type):
    """max_q 0 says nothing of the longest sequence: the places of both kernels are in the workspace, as with the true
    max_q."""
    T, B, keys = sum(new), len(new), 16384
    unknown, true, few = (workspace(B, T, keys, Hq, Hkv, type=type, max_q=q, path=path)
                          for q, path in ((0, fa.FA_PAGED_AUTO), (max(new), fa.FA_PAGED_AUTO), (max(new), fa.FA_PAGED_FEW)))
    if (B, Hkv) == (25, 8) and type == 0:
        assert few < true  # a chunk's blocks are split: their places too
    assert unknown == true > 0


@pytest.mark.parametrize("n,B", [(1, 1), (1, 64), (5, 8), (9, 16), (2, 64)])
def test_without_max_q_few_tokens_are_taken_for_what_they_are(n, B):
    """Too few tokens for the kernel for many rows however they lie: planned as with the true max_q."""
    for heads in ((32, 8), (14, 2), (8, 1)):
        assert workspace(B, n * B, 2000, *heads, max_q=0, path=0) == workspace(B, n * B, 2000, *heads, max_q=n, path=1)
    assert workspace(1, 4096, 4096, 32, 8, max_q=0, path=0) == workspace(1, 4096, 4096, 32, 8, max_q=4096, path=0)
