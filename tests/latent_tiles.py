"""Queries of the latent attention whose results say which slots were read, and how often.

A query that is the sum of two slots' rows, each over its own square, has their scores at `aim` and all others near zero: its result is
half of either latent.  With a slot lost it is the other's alone, with one read twice it lies at two thirds, with one in another's place it is
neither: a sixth of the latents' difference at least, where roundings are a hundredth of the latents."""
import torch

AIM = 30.0


def paired_queries(rows, pairs, scale):
    """rows [slots, D]; pairs [n, 2] of slots -> [n, D] in rows' type."""
    r = rows.double()[pairs]
    return ((r / r.square().sum(-1, keepdim=True)).sum(1) * (AIM / scale)).to(rows.dtype)


def pairs_over(slots, tile, seed):
    """Every tile's slots in turn first, last or somewhere in it, in an order that puts far ones together: [ceil(tiles / 2), 2]."""
    g = torch.Generator().manual_seed(seed)
    tiles = -(-slots // tile)
    at = torch.arange(tiles)
    off = torch.randint(0, tile, (tiles,), generator=g)
    off[at % 3 == 0], off[at % 3 == 1] = 0, tile - 1
    s = torch.minimum(at * tile + off, torch.tensor(slots - 1))[torch.randperm(tiles, generator=g)]
    if tiles % 2:
        s = torch.cat([s, s[:1]])
    return s.view(-1, 2)


def rms_off(got, y):
    """Relative distance over all of a call's results.  A rounding to bf16 is off by a value's step times at most a half, evenly spread,
    over values whose logarithm is: 2^-8 / sqrt(3) * sqrt(3 / (8 ln 2)) = 0.00166 of the value, root of the mean square.  Results are rounded once;
    the softmax's weights too, independent of each other and of the latents, which leaves at most as much again of a result whose latents
    have no mean: sqrt(2) * 0.00166 = 0.0024, and float32's part is below 10^-4 of that.  0.003 leaves a quarter for the spread."""
    got, y = got.double(), y.double()
    return ((got - y).norm() / y.norm()).item()


RMS = 0.003
