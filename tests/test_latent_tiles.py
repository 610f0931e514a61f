"""What the queries of latent_tiles.py find, on the CPU: mistakes planted in a float64 attention."""
import pytest
import torch

from latent_tiles import RMS, paired_queries, pairs_over, rms_off

U = 2.0 ** -8
TILE = 32


def attend(q, rows, c, scale, order=None, count=None):
    """Attention over rows[order], slot i of them counted count[i] times."""
    k = rows if order is None else rows[order]
    p = torch.exp(q @ k.T * scale - (q @ rows.T * scale).amax(-1, keepdim=True)) * (1.0 if count is None else count)
    return (p @ k[:, :c]) / p.sum(-1, keepdim=True), (p @ k[:, :c].abs()) / p.sum(-1, keepdim=True)


@pytest.mark.parametrize("c,r,slots", [(512, 64, 1000), (512, 64, 7001), (256, 32, 3003)])
def test_a_tile_lost_doubled_or_misplaced_shows(c, r, slots):
    scale = (c // 4 + r) ** -0.5
    rows = torch.randn(slots, c + r, generator=torch.Generator().manual_seed(slots)).to(torch.bfloat16)
    pairs = pairs_over(slots, TILE, 1)
    assert torch.equal(torch.unique(pairs // TILE), torch.arange(-(-slots // TILE)))
    q, rows = paired_queries(rows, pairs, scale).double(), rows.double()
    y, mag = attend(q, rows, c, scale)
    off = U * y.abs() + 1.1 * U * mag                                   # the roundings that a right kernel has
    rounded = y.to(torch.bfloat16)
    assert ((rounded - y).abs() <= off).all() and rms_off(rounded, y) <= RMS
    for tile in range(0, -(-slots // TILE), 3):
        mine = (pairs // TILE == tile).any(-1) & (pairs[:, 0] != pairs[:, 1])
        if not mine.any():
            continue
        lo, hi = tile * TILE, min((tile + 1) * TILE, slots)
        kept = torch.ones(slots, dtype=torch.double)
        kept[lo:hi] = 0
        twice = kept.clone()
        twice[lo:hi] = 2
        other = torch.arange(slots)
        other[lo:hi] = (torch.arange(lo, hi) + TILE) % slots
        for order, count in ((None, kept), (None, twice), (other, None)):
            wrong, _ = attend(q[mine], rows, c, scale, order, count)
            assert ((wrong - y[mine]).abs() > off[mine]).double().mean(-1).min() > 0.5
            assert rms_off(wrong, y[mine]) > 10 * RMS


def test_a_right_kernels_roundings_are_within():
    """Weights rounded to bf16 over their own sum, results rounded once: as much as rms_off says."""
    c, r, slots = 512, 64, 5000
    scale = (c // 4 + r) ** -0.5
    g = torch.Generator().manual_seed(4)
    rows = torch.randn(slots, c + r, generator=g).to(torch.bfloat16).double()
    q = torch.randn(32, c + r, generator=g).to(torch.bfloat16).double()
    p = torch.exp(q @ rows.T * scale - (q @ rows.T * scale).amax(-1, keepdim=True))
    w = p.to(torch.bfloat16).double()
    got = ((w @ rows[:, :c]) / w.sum(-1, keepdim=True)).to(torch.bfloat16)
    assert 0.5 * RMS <= rms_off(got, (p @ rows[:, :c]) / p.sum(-1, keepdim=True)) <= RMS
