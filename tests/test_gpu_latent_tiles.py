"""Every tile of a latent attention's range is read once, in its place: long contexts, many chunks, pages, batches."""
import pytest
import torch

import paper_2504_04104_amd as sp
from latent_reference import attend, make, seen_by
from latent_tiles import RMS, paired_queries, pairs_over, rms_off
from test_gpu_latent import check_rows, rnd

pytestmark = pytest.mark.gpu
LONG = [(1, 20000, 1), (16, 40000, 1), (16, 32749, 5), (128, 9000, 2), (64, 16383, 20), (8, 70000, 3), (64, 4096, 128), (16, 513, 1), (3, 100, 7)]


def check_all(st, heads, c, r, scale, calls_of):
    """calls_of(i) -> (pairs, first committed slots) of request i; every request's queries spread over as many calls as they take."""
    n = [T for _, T in st.trees]
    qs = [paired_queries(st.held[i], calls_of(i).cuda(), scale) for i in range(len(n))]
    calls = max(-(-len(q) // (heads * T)) for q, T in zip(qs, n))
    filled = [q.repeat(-(-calls * heads * T // len(q)), 1)[:calls * heads * T].view(calls, T, heads, c + r) for q, T in zip(qs, n)]
    ids = list(range(len(n)))
    got = [st.attention(0, ids, [0] * len(n), n, torch.cat([f[k] for f in filled])).split(n) for k in range(calls)]
    for i in ids:
        y = torch.cat([g[i] for g in got])
        check_rows(y, filled[i].flatten(0, 1), st.held[i], c, seen_by(st, i).repeat(calls, 1), scale)
        want = attend(filled[i].flatten(0, 1), st.held[i], c, seen_by(st, i).repeat(calls, 1), scale)[0]
        assert rms_off(y, want) <= RMS, i


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("heads,P,T", LONG)
def test_every_tile_of_a_long_context(heads, P, T, page):
    st = make(heads, 512, 64, [(P, T)], page=page, scale=0.07)
    check_all(st, heads, 512, 64, 0.07, lambda i: pairs_over(P, 32, P))


@pytest.mark.parametrize("c,r", [(256, 32), (512, 32), (256, 64)])
def test_every_tile_of_other_spaces(c, r):
    for heads, P, T in ((16, 20001, 2), (128, 3000, 3)):
        st = make(heads, c, r, [(P, T)], scale=0.07)
        check_all(st, heads, c, r, 0.07, lambda i: pairs_over(P, 32, P))


@pytest.mark.parametrize("page", [0, 32, 256])
def test_every_tile_of_a_batch(page):
    trees = [(300 + 131 * i, 1 + i % 5) for i in range(32)]
    st = make(16, 512, 64, trees, page=page, scale=0.07)
    check_all(st, 16, 512, 64, 0.07, lambda i: pairs_over(trees[i][0], 32, i))


def test_every_tile_by_plain_kernels():
    st = make(8, 512, 64, [(4000, 3)], scale=0.07, flags=sp.SP_FLAG_SIMPLE_KERNELS)
    check_all(st, 8, 512, 64, 0.07, lambda i: pairs_over(4000, 32, 5))


@pytest.mark.parametrize("heads,P,T", LONG[:7])
def test_random_queries_are_off_by_roundings_alone(heads, P, T):
    st = make(heads, 512, 64, [(P, T)])
    q, scale = rnd(7, T, heads, 576), (128 + 64) ** -0.5
    y = st.attention(0, [0], [0], [T], q)
    assert rms_off(y, attend(q, st.held[0], 512, seen_by(st, 0), scale)[0]) <= RMS
