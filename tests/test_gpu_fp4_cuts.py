"""Products with 4-bit weights through every kernel and cut of them (fp4_cases.py), as calls of their own and inside the forward
call, against float64 on the values held.  (test_gpu_fp4.py pins the held values themselves.)"""
import pytest
import torch

import paper_2504_04104_amd as sp
import workloads as wl
from fp4_cases import FORWARDS, PRODUCTS
from fp4_layers import layer, matrix, tree
from fp4_reference import random_tree, stage

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -8, 2.0 ** -24                        # half a step of bf16 and of float32, relative to the value


def rnd(seed, *size, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*size, generator=g, device="cuda", dtype=torch.bfloat16) * scale


@pytest.mark.parametrize("m,n,k,gated", PRODUCTS)
def test_product(m, n, k, gated):
    """Off by the result's rounding and float32 sums of k terms in any order: at most k * 2^-24 times the sum of their magnitudes.
    silu changes by at most 1.1 per unit, and its exponential and quotient are good to 2^-20."""
    x, p = rnd(m, m, k), sp.fp4_pack_matrix(rnd(n, n * (2 if gated else 1), k, scale=0.05))
    y, w, xd = sp.fp4_product(x, p, gated=gated).double(), matrix(p), x.double()
    ref, mag = xd @ w.T, k * F * (xd.abs() @ w.abs().T)
    if gated:
        a, b, ea, eb = ref[:, :n], ref[:, n:], mag[:, :n], mag[:, n:]
        s = a * torch.sigmoid(a)
        ref, mag = s * b, 1.1 * ea * (b.abs() + eb) + s.abs() * eb + 2.0 ** -20 * (s * b).abs()
    assert y.shape == ref.shape
    assert ((y - ref).abs() <= U * ref.abs() + 1.01 * mag + 1e-30).all()


@pytest.mark.parametrize("d,nq,nkv,ff,m", FORWARDS)
def test_forward(d, nq, nkv, ff, m):
    """The float64 layer rounds where the framework keeps bfloat16: scores of some hundred, as wide layers make them here, move
    by more than one for what queries and keys are rounded by, and the layer with no rounding in it is up to 3.85 % of the largest
    value from the one with (d = 5632, 195 rows).  What is left to differ is the order of float32 sums, the softmax's weights, and
    roundings that those turn: half of the bar of the other forward calls."""
    sh = wl.ModelShape(1, d, nq, nkv, 128, ff, 1e-5, 500000.0, "bf16")
    size = {"wqkv": ((nq + 2 * nkv) * 128, d), "wo": (d, nq * 128), "wgu": (2 * ff, d), "wd": (d, ff)}
    w = {name: rnd(i, *s, scale=0.05) for i, (name, s) in enumerate(size.items())}
    for i, name in enumerate(("norm1", "norm2")):
        w[name] = 1 + rnd(8 + i, d, scale=0.05)
    st = stage(sp, sh, slots=512, flags=sp.SP_FLAG_FP4_WEIGHTS, rows=256, layers=[w])
    del w
    P, parents = (1 if m % 2 else 51), random_tree(m, m)
    st.request_init(0, 0, 400, P)
    k, v = rnd(20, P, nkv, 128), rnd(21, P, nkv, 128)
    st.kv_store(0, 0, 0, k, v)
    st.tree_insert(0, parents)
    x = rnd(22, m, d)
    y = st.stage_forward([0], [0], [m], x).double()
    pos, seen = tree(P, parents)
    ref = layer(st.layers[0], x.double(), pos, seen, lambda kn, vn: (torch.cat([k.double(), kn]), torch.cat([v.double(), vn])), sh)
    assert (y - ref).abs().max() <= 1e-2 * ref.abs().max()
    assert ((y - x.double()) - (ref - x.double())).abs().max() <= 2e-2 * (ref - x.double()).abs().max()
