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


def test_partial_rows_only_where_ranges_are_cut():
    """Matrix-core kernels: room for 40960 partial rows of d_latent + 2 floats.  Plain kernels cut nothing: room for the output head
    alone, which a latent's size does not change."""
    def workspace(**kw):
        rc, sz = sizes(**kw)
        assert rc == OK
        return sz.workspace_bytes
    head = workspace(c=8, r=8)
    for c, r in ((512, 64), (512, 32), (256, 64), (256, 32)):
        assert workspace(c=c, r=r) == head + 40960 * (c + 2) * 4
        assert workspace(c=c, r=r, flags=sp.SP_FLAG_SIMPLE_KERNELS) == head
    for c, r in ((1024, 128), (512, 128), (136, 64), (1024, 8)):
        assert workspace(c=c, r=r) == workspace(c=c, r=r, flags=sp.SP_FLAG_SIMPLE_KERNELS) == head
