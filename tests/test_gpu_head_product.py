"""Products head by head against float64.  u = 2^-8 is half a step of bf16 relative to the value; a float32 sum of k products in any order
is off by at most k * 2^-24 times the sum of their magnitudes."""
import pytest
import torch

import paper_2504_04104_amd as sp
from gpu_harness import use_own_stream

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -8, 2.0 ** -24


def rnd(seed, *size, scale=1.0):
    return (scale * torch.randn(*size, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda()


def near(y, x, w):
    k = x.shape[-1]
    for h in range(x.shape[1]):
        a, b = x[:, h].double(), w[h].double()
        ref, mag = a @ b.T, a.abs() @ b.abs().T
        assert ((y[:, h].double() - ref).abs() <= U * ref.abs() + 1.01 * k * F * mag + 1e-30).all(), h


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 100, 127, 129, 257, 640])
@pytest.mark.parametrize("n,k", [(512, 128), (128, 512), (256, 64), (64, 256), (16, 32)])
def test_any_number_of_rows(m, n, k):
    x, w = rnd(m, m, 5, k), rnd(n, 5, n, k, scale=k ** -0.5)
    near(sp.head_product(x, w), x, w)


@pytest.mark.parametrize("m,heads,n,k", [(1, 1, 16, 32), (3, 128, 512, 128), (70, 3, 48, 96), (5, 2, 4096, 4096), (9, 1, 1040, 608), (130, 2, 272, 1056),
                                         (1, 200, 16, 4096), (20000, 1, 64, 64), (2, 4096, 16, 32), (33, 7, 80, 160)])
def test_many_shapes(m, heads, n, k):
    x, w = rnd(m, m, heads, k), rnd(n, heads, n, k, scale=k ** -0.5)
    near(sp.head_product(x, w), x, w)


@pytest.mark.parametrize("m", [1, 5, 64, 200])
def test_views(m):
    """Part of the columns of wider rows, into part of the columns of others; heads one behind the other; a row for all."""
    q, w = rnd(1, m, 6, 192), rnd(2, 6, 256, 128, scale=0.1)
    wide = torch.full((m + 1, 6, 288), 3.0, dtype=torch.bfloat16, device="cuda")
    sp.head_product(q[..., :128], w, out=wide[:m, :, :256])
    near(wide[:m, :, :256], q[..., :128], w)
    assert (wide[:, :, 256:] == 3).all() and (wide[m] == 3).all()
    major = torch.zeros(6, m, 256, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(sp.head_product(q[..., :128], w, out=major), wide[:m, :, :256])
    same = rnd(3, 1, 1, 128).expand(m, 6, 128)
    near(sp.head_product(same, w), same, w)


def test_what_is_not_finite_stays_in_its_row():
    x, w = rnd(1, 40, 3, 128), rnd(2, 3, 64, 128)
    clean = sp.head_product(x, w)
    x[7, 1, 5] = float("nan")
    x[20, 2, 0] = float("inf")
    y = sp.head_product(x, w)
    assert torch.isnan(y[7, 1]).all() and not torch.isfinite(y[20, 2]).any()
    y[7, 1], y[20, 2] = clean[7, 1], clean[20, 2]
    assert torch.equal(y, clean)


def test_a_captured_product_replays():
    use_own_stream()
    x, w = rnd(1, 20, 4, 128), rnd(2, 4, 512, 128)
    out = torch.zeros(20, 4, 512, dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.head_product(x, w, out=out)
    for k in range(3):
        x.copy_(rnd(10 + k, 20, 4, 128))
        g.replay()
        assert torch.equal(out, sp.head_product(x, w))


def test_refusals():
    x, w = rnd(1, 4, 2, 64), rnd(2, 2, 32, 64)

    def refused(status, call):
        with pytest.raises(sp.SpError) as err:
            call()
        assert err.value.status == status
    refused(-9, lambda: sp.head_product(rnd(1, 4, 2, 48), rnd(2, 2, 32, 48)))
    refused(-9, lambda: sp.head_product(x, rnd(2, 2, 24, 64)))
    both = torch.zeros(4, 2, 96, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: sp.head_product(both[..., :64], w, out=both[..., 64:]))
    refused(-9, lambda: sp.head_product(x, w, out=torch.zeros(4, 1, 32, dtype=torch.bfloat16, device="cuda").expand(4, 2, 32)))
    refused(-9, lambda: sp.head_product(rnd(1, 4, 2, 68)[..., :64], w))
    assert sp.head_product(x[:0], w).shape == (0, 2, 32)


@pytest.mark.parametrize("heads,n,k", [(16, 512, 128), (33, 512, 128), (64, 128, 512), (128, 64, 96)])
@pytest.mark.parametrize("m", [1, 16, 17, 64, 65, 256, 449])
def test_few_heads_and_many(m, heads, n, k):
    """Either side of where the rows of a block and the columns of a workgroup change."""
    x, w = rnd(m, m, heads, k), rnd(n, heads, n, k, scale=k ** -0.5)
    near(sp.head_product(x, w), x, w)


@pytest.mark.parametrize("heads,n,k", [(40, 320, 64), (64, 64, 64), (24, 512, 128), (48, 192, 128), (32, 192, 192), (16, 1024, 256)])
@pytest.mark.parametrize("m", [97, 641, 2049])
def test_columns_kept_for_many_rows(m, heads, n, k):
    """Columns that end inside a workgroup, rows inside a block; workgroups with one block and with more."""
    x, w = rnd(m, m, heads, k), rnd(n, heads, n, k, scale=k ** -0.5)
    near(sp.head_product(x, w), x, w)


@pytest.mark.parametrize("k", [64, 128, 192, 256])
def test_views_of_many_rows(k):
    m, heads, n = 1100, 32, 320
    q, w = rnd(1, m + 1, heads, k + 24), rnd(2, heads, n, k, scale=0.1)
    wide = torch.full((m + 1, heads, n + 40), 3.0, dtype=torch.bfloat16, device="cuda")
    sp.head_product(q[:m, :, 8:k + 8], w, out=wide[:m, :, 8:n + 8])
    near(wide[:m, :, 8:n + 8], q[:m, :, 8:k + 8], w)
    assert (wide[m] == 3).all() and (wide[..., :8] == 3).all() and (wide[..., n + 8:] == 3).all()
    one = q[:1, :, :k].expand(m, heads, k)
    got = sp.head_product(one, w)
    assert torch.equal(got, got[:1].expand(m, heads, n))
    near(got[:1], one[:1], w)
