"""Columns that a stage's rotation leaves out pass: as they came, whatever stands in them or beside them."""
import numpy as np
import pytest
import torch

import workloads as wl
import paper_2504_04104_amd as sp
from fp4_reference import stage
from gpu_harness import use_own_stream

pytestmark = pytest.mark.gpu
SHAPES = {"bf16_128": ((8, 2, 128), "bf16"), "bf16_64": ((4, 4, 64), "bf16"), "f32_64": ((4, 2, 64), "f32")}


def same(a, b):
    """Equal values and signs of zeros, NaN where there is NaN."""
    a, b = a.float(), b.float()
    nan = torch.isnan(b)
    return torch.equal(torch.isnan(a), nan) and torch.equal(a[~nan], b[~nan]) and torch.equal(torch.signbit(a[~nan]), torch.signbit(b[~nan]))


@pytest.mark.parametrize("layout,part", [("half", 2), ("interleaved", 2), ("interleaved", 8)])
@pytest.mark.parametrize("cache", sorted(SHAPES))
def test_appended_heads(cache, layout, part):
    (nq, kv, dh), dtype = SHAPES[cache]
    st = stage(sp, wl.ModelShape(1, 256, nq, kv, dh, 256, 1e-5, 500000.0, dtype), slots=256, rows=64)
    st.request_init(0, 0, 200, 100)
    st.tree_insert(0, [-1, 0, 1, 1, 3])
    dims = dh // part
    st.set_rope(sp.Rope(layout, dims, 10000.0, gain=1.1))
    x = torch.randn(5, nq + 2 * kv, dh, generator=torch.Generator().manual_seed(dims)).to("cuda", st.tdtype)
    clean = st.append(0, [0], [0], [5], x.reshape(5, -1)).reshape(5, nq, dh), st.kv_load(0, 0, 100, 5)[0].reshape(5, kv, dh)
    for col in (dims, dims + 1, dims + 4, dh - 2, dh - 1):
        for bad in (float("inf"), -float("inf"), float("nan"), -0.0):
            h = x.clone()
            h[:, :, col] = bad
            h[:, :, col ^ 1] = -h[:, :, col ^ 1].abs()                      # (beside a negative zero: products of either sign)
            q = st.append(0, [0], [0], [5], h.reshape(5, -1)).reshape(5, nq, dh)
            k = st.kv_load(0, 0, 100, 5)[0].reshape(5, kv, dh)
            assert same(q[..., dims:], h[:, :nq, dims:]) and same(k[..., dims:], h[:, nq:nq + kv, dims:]), (col, bad)
            assert same(q[..., :dims], clean[0][..., :dims]) and same(k[..., :dims], clean[1][..., :dims]), (col, bad)


@pytest.mark.parametrize("dtype,n", [("bf16", 3), ("bf16", 40), ("bf16", 200), ("f32", 9)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_forward_calls(dtype, n, layout):
    """A key column whose weights hold an infinity: every other column of the cached keys is as without it."""
    use_own_stream()
    dh, nq, kv, d = (128, 4, 2, 512) if dtype == "bf16" else (64, 4, 2, 256)
    sh = wl.ModelShape(1, d, nq, kv, dh, 512, 1e-5, 500000.0, dtype)
    x = torch.randn(n, d, generator=torch.Generator().manual_seed(n)).to("cuda", torch.bfloat16 if dtype == "bf16" else torch.float32)
    keys = []
    for col in (None, dh - 2, dh // 2 + 1):
        plain = stage(sp, sh, slots=512, rows=256).plain_layers
        if col is not None:
            plain[0]["wqkv"][nq * dh + col, 7] = float("inf")
        st = stage(sp, sh, slots=512, rows=256, layers=plain)
        st.request_init(0, 0, 500, 30)
        st.tree_insert(0, [-1] * n)
        st.set_rope(sp.Rope(layout, dh // 2, 10000.0))
        st.stage_forward([0], [0], [n], x)
        k = st.kv_load(0, 0, 30, n)[0].reshape(n, kv, dh)
        if col is None:
            keys = k
            continue
        assert not torch.isfinite(k[:, 0, col]).any()
        rest = np.arange(dh) != col
        assert same(k[:, 0, rest], keys[:, 0, rest]) and same(k[:, 1], keys[:, 1])
