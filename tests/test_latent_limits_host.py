"""Limits of a latent stage's sizes, asked for without a GPU."""
import pytest

import paper_2504_04104_amd as sp
from test_latent_host import OK, UNSUPPORTED, sizes


@pytest.mark.parametrize("c,r", [(8, 8), (512, 64)])
def test_slots_that_32_bits_count_with_a_tile_to_spare(c, r):
    """The plain kernel takes 256 slots at a time, the split rounds ranges up to chunks: at 2^31 - 1 slots, which 64 GB hold in the
    smallest space, either would count past 2^31 and go on from below zero."""
    assert sizes(c=c, r=r, slots=1 << 30)[0] == OK
    for slots in ((1 << 30) + 1, (1 << 31) - 257, (1 << 31) - 1):
        assert sizes(c=c, r=r, slots=slots)[0] == UNSUPPORTED, slots
        page = dict(flags=sp.SP_FLAG_PAGED_KV, page=32, slots=slots // 32 * 32)
        if page["slots"] > 1 << 30:
            assert sizes(c=c, r=r, **page)[0] == UNSUPPORTED, slots
