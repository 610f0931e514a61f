"""What the 4-bit entry points refuse and say without touching a GPU, and the float64 reference of the format itself."""
import ctypes as C

import numpy as np
import pytest

import paper_2504_04104_amd as sp
from paper_2504_04104_amd import binding
from fp4_reference import GRID, group_exponent, held

OK, INVALID, CAPACITY, UNSUPPORTED = 0, -1, -2, -9


def cfg(dtype=binding.SP_BF16, d_head=128, flags=0, page=0, slots=2560):
    return binding.sp_config(4, 4096, 32, 8, d_head, 14336, 1e-5, 500000.0, dtype, 1, 256, 64, slots, flags, page)


def sizes(c):
    sz = binding.sp_sizes()
    return sp.load_library().sp_stage_query_sizes(C.byref(c), C.byref(sz)), sz


def test_sizes_of_a_cache_in_4_bits():
    for dh in (64, 128):
        rc, sz = sizes(cfg(d_head=dh, flags=sp.SP_FLAG_FP4_KV))
        assert rc == OK and sz.kv_row_bytes == dh // 2 and sz.kv_plane_bytes == 2560 * dh // 2
        assert sz.kv_bytes == 4 * 2 * 8 * 2560 * (dh // 2 + 4)
    assert sizes(cfg(flags=sp.SP_FLAG_FP4_KV | sp.SP_FLAG_PAGED_KV, page=64))[0] == OK
    assert sizes(cfg(dtype=binding.SP_F32, flags=sp.SP_FLAG_FP4_KV))[0] == UNSUPPORTED
    assert sizes(cfg(dtype=binding.SP_F32, flags=sp.SP_FLAG_FP4_WEIGHTS))[0] == UNSUPPORTED
    assert sizes(cfg(flags=sp.SP_FLAG_FP4_WEIGHTS | sp.SP_FLAG_PACKED_WEIGHTS))[0] == INVALID
    # what other stages need is what they needed
    assert sizes(cfg())[1].kv_bytes == 4 * 2 * 8 * 2560 * 256


def test_bytes_of_packed_matrices():
    f = sp.load_library().sp_fp4_matrix_bytes
    assert f(16, 256) == 2176 and f(16, 32) == 2176 and f(32, 288) == 2 * 2 * 2176
    assert f(28672, 8192) == 28672 * 8192 * 17 // 32
    for n, k in ((0, 32), (-16, 32), (17, 32), (16, 16), (16, 33), (16, 0), (16, -32), (1 << 18, 32), (16, 1 << 18), (2 ** 31 - 16, 32)):
        assert f(n, k) == 0, (n, k)


def test_refused_products_and_matrices():
    lib = sp.load_library()
    p = [C.c_void_p(4096 * (i + 1)) for i in range(4)]                 # never read: every call below is refused first
    odd = C.c_void_p(4104)

    def product(x=p[0], m=1, w=p[1], n=16, k=32, gated=0, out=p[2], work=None, size=0):
        return lib.sp_fp4_product(x, m, w, n, k, gated, out, work, size, None)

    for bad in (dict(x=None), dict(w=None), dict(out=None), dict(m=-1), dict(n=0), dict(k=0), dict(n=-16), dict(gated=2), dict(gated=-1), dict(x=odd),
                dict(w=odd), dict(out=odd), dict(work=odd)):
        assert product(**bad) == INVALID, bad
    for bad in (dict(n=17), dict(k=48), dict(n=8, gated=1), dict(n=1 << 17, gated=1), dict(k=1 << 18), dict(m=(1 << 17) + 1), dict(n=2 ** 31 - 16)):
        assert product(**bad) == UNSUPPORTED, bad
    need = lib.sp_fp4_product_workspace(1, 16, 8192, 0)
    assert need > 0
    assert product(k=8192) == CAPACITY and product(k=8192, work=p[3], size=need - 1) == CAPACITY
    assert product(m=0) == OK
    assert lib.sp_fp4_product_workspace(1, 17, 32, 0) == 0 and lib.sp_fp4_product_workspace(-1, 16, 32, 0) == 0
    for f in (lib.sp_fp4_pack_matrix, lib.sp_fp4_unpack_matrix):
        assert f(None, p[1], 16, 32, None) == INVALID and f(p[0], None, 16, 32, None) == INVALID and f(p[0], p[0], 16, 32, None) == INVALID
        assert f(odd, p[1], 16, 32, None) == INVALID and f(p[0], p[1], 0, 32, None) == INVALID
        assert f(p[0], p[1], 8, 32, None) == UNSUPPORTED and f(p[0], p[1], 16, 40, None) == UNSUPPORTED
    a, b = binding.sp_layer_weights(), binding.sp_layer_weights()
    assert lib.sp_fp4_pack_weights(C.byref(cfg()), C.byref(a), C.byref(b), None) == INVALID
    assert lib.sp_fp4_pack_weights(C.byref(cfg(dtype=binding.SP_F32)), C.byref(a), C.byref(b), None) == UNSUPPORTED


def test_calls_without_a_stage():
    lib = sp.load_library()
    one = (C.c_int32 * 1)(0)
    p = C.c_void_p(4096)
    assert lib.sp_kv_store(None, 0, 0, 0, 1, p, p, None) == INVALID
    assert lib.sp_kv_load(None, 0, 0, 0, 1, p, p, None) == INVALID
    assert lib.sp_stage_set_head_norms(None, None) == INVALID
    assert lib.sp_stage_append(None, 0, 1, one, one, one, p, p, None) == INVALID
    assert lib.sp_stage_attention(None, 0, 1, one, one, one, p, p, None) == INVALID


def test_reference_holds_the_nearest_grid_value():
    r = np.random.default_rng(0)
    x = r.standard_normal((50, 64)) * 2.0 ** r.integers(-20, 20, (50, 1))
    e = group_exponent(x)
    g = np.abs(x).reshape(50, 2, 32)
    assert (g.max(-1) <= 6 * 2.0 ** e).all() and (g.max(-1) > 6 * 2.0 ** (e - 1)).all()
    a = g / 2.0 ** e[..., None]
    best = np.abs(a[..., None] - GRID).min(-1)
    assert np.allclose(np.abs(np.abs(held(x)).reshape(g.shape) / 2.0 ** e[..., None] - a), best)
    ties = np.zeros((1, 32))
    ties[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0]
    assert held(ties)[0, :8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -6.0]
