"""Infinities in cache rows of the latent attention that a query row sees.

A score of minus infinity is a weight of zero: its slot counts as nothing, whatever it holds.  A score of plus infinity, or one that is
no number, makes the query row's whole result NaN.  So it is in every kernel, tile and chunk, in the committed context and the tree."""
import math

import pytest
import torch

import paper_2504_04104_amd as sp
from latent_reference import make, seen_by
from test_gpu_latent import check_rows, rnd

pytestmark = pytest.mark.gpu
SCALE = 0.07


def check_call(got, q, rows, c, seen):
    """Rows of the call by what they see: NaN, or the attention over the slots whose score is not minus infinity."""
    score = torch.einsum("nhd,sd->nhs", q.double().cpu(), rows.double().cpu()).cuda()
    lost = torch.isneginf(score) & seen[:, None]
    none = ((torch.isnan(score) | torch.isposinf(score)) & seen[:, None]).any(-1) | ~(seen[:, None] & ~lost).any(-1)
    clean = torch.where(torch.isfinite(rows), rows, torch.zeros_like(rows))
    for h in range(q.shape[1]):
        assert torch.isnan(got[none[:, h], h]).all()
        ok = ~none[:, h]
        if ok.any():
            check_rows(got[ok, h:h + 1], q[ok, h:h + 1], clean, c, (seen & ~lost[:, h])[ok], SCALE)
    return int(none.sum()), int((lost.any(-1) & ~none).sum())


CASES = [(16, 512, 64, 700, 5, 0), (64, 512, 64, 700, 40, 0), (5, 256, 32, 700, 5, 0), (16, 512, 64, 9000, 3, 0), (16, 512, 64, 9000, 3, 64),
         (128, 512, 32, 1500, 20, 0), (3, 256, 64, 61, 2, 0)]


@pytest.mark.parametrize("flags", [0, sp.SP_FLAG_SIMPLE_KERNELS])
@pytest.mark.parametrize("heads,c,r,P,T,page", CASES)
def test_slots_with_an_infinity(heads, c, r, P, T, page, flags):
    nothing = whole = 0
    for slots in ([5], [P // 2], [P // 2, P // 2 + 17], [P - 1], [P], [P + T - 1], [0, P // 3, P]):
        for col, bad in ((1, math.inf), (c - 1, -math.inf), (c + 3, math.inf)):
            st = make(heads, c, r, [(P, T)], page=page, flags=flags, scale=SCALE, seed=P)
            rows, q = st.held[0].clone(), rnd(3, T, heads, c + r)
            q[0, 0, col] = 0.0                                              # (zero times infinity)
            rows[slots, col] = bad
            st.kv_store(0, 0, 0, rows)
            n, m = check_call(st.attention(0, [0], [0], [T], q), q, rows, c, seen_by(st, 0))
            whole, nothing = whole + n, nothing + m
    assert whole > 0 and nothing > 0


@pytest.mark.parametrize("flags", [0, sp.SP_FLAG_SIMPLE_KERNELS])
@pytest.mark.parametrize("heads,P", [(4, 300), (16, 5000)])
def test_a_context_that_counts_as_nothing(heads, P, flags):
    """Every committed slot at minus infinity: the nodes alone are left; with theirs too, nothing, which is NaN."""
    T, c = 3, 512
    st = make(heads, c, 64, [(P, T)], flags=flags, scale=SCALE)
    rows, q = st.held[0].clone(), rnd(3, T, heads, 576)
    q[..., 2] = q[..., 2].abs() + 0.1
    for to in (P - 1, P, P + T):
        rows[:to, 2] = -math.inf
        st.kv_store(0, 0, 0, rows)
        check_call(st.attention(0, [0], [0], [T], q), q, rows, c, seen_by(st, 0))


def test_replayed_and_repeated_calls_have_equal_bits():
    """A slot whose values are taken out of a tile is taken out of the workgroup's copy, not of the cache."""
    st = make(16, 512, 64, [(3000, 5)], scale=SCALE)
    rows, q = st.held[0].clone(), rnd(3, 5, 16, 576)
    rows[[40, 1500, 2999, 3001], 9] = math.inf
    st.kv_store(0, 0, 0, rows)
    first = st.attention(0, [0], [0], [5], q)
    for _ in range(5):
        again = st.attention(0, [0], [0], [5], q)
        assert torch.equal(again.view(torch.int16), first.view(torch.int16))
    assert torch.equal(st.kv_load(0, 0, 0, 3005), rows)
