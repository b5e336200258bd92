"""Counts at the borders of what the moves around the paged cache launch, on the host (no GPU needed)."""

import pytest

import paper_2609_21264_amd as fa
from test_cache_moves_host import NULL, SHAPE, append_at, batch, cache, compact
from test_paged_host import append


@pytest.mark.parametrize("Hkv,blocks", [(1, 1), (8, 1), (9, 2), (4096, 512)])
def test_compact_of_more_workgroups_than_a_copy(Hkv, blocks):
    """A workgroup moves 256 chunks of 16 bytes of a sequence's tokens, a token's K and V in d = 128, bf16 being 32 a head:
    fewer than 2^24 workgroups in all, as in a copy of pages. Behind 2^31 the kernel's number of a sequence would wrap."""
    c = cache(Hkv=Hkv, k_page=Hkv * 16 * 128, v_page=Hkv * 16 * 128)
    most = (2 ** 24 - 1) // blocks
    assert compact(c, batch(B=most), n_kept=None) == NULL  # sizes are right
    for B in (most + 1, 2 ** 30, 2 ** 31 - 32768, 2 ** 31 - 65, 2 ** 31 - 2):
        assert compact(c, batch(B=B), n_kept=None) == SHAPE, B


@pytest.mark.parametrize("call", [append, append_at])
def test_append_to_as_many_sequences_as_32_bits_count(call):
    """The search for a token's sequence rounds the number of starts, B + 1, up to a multiple of 64."""
    assert call(b=batch(B=2 ** 31 - 65), K=None) == NULL  # sizes are right
    for B in (2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 2, 2 ** 31 - 1):
        assert call(b=batch(B=B), K=None) == SHAPE, B


def test_a_softcap_that_float32_does_not_hold():
    """What rounds to 0 would be no cap at all; what float32 holds, down to its smallest number, is one."""
    none = None, None, None, None, 1, 4, 1, 0
    for cap in (1e-46, 1e-50, 5e-324):
        with pytest.raises(ValueError, match="softcap must be above 0"):
            fa._scores(cap, *none)
    for cap in (1e-45, 1e-30, 1, 1024.0):
        assert fa._scores(cap, *none).softcap > 0
