"""What the 4-bit entry points refuse and say without touching a GPU, and the float64 reference of the format itself."""
import ctypes as C
import os
import subprocess

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
    most = (1 << 25) - 1                            # a plane of codes stays under 2 GB
    assert sizes(cfg(slots=most, flags=sp.SP_FLAG_FP4_KV))[0] == OK
    assert sizes(cfg(slots=most + 1, flags=sp.SP_FLAG_FP4_KV))[0] == UNSUPPORTED
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
    p = [C.c_void_p((i + 1) << 24) for i in range(4)]                  # never read: every call below is refused first
    odd = C.c_void_p(4104)

    def product(x=p[0], m=1, w=p[1], n=16, k=32, gated=0, out=p[2], work=None, size=0):
        return lib.sp_fp4_product(x, m, w, n, k, gated, out, work, size, None)

    for bad in (dict(x=None), dict(w=None), dict(out=None), dict(m=-1), dict(n=0), dict(k=0), dict(n=-16), dict(gated=2), dict(gated=-1), dict(x=odd),
                dict(w=odd), dict(out=odd), dict(work=odd)):
        assert product(**bad) == INVALID, bad
    for bad in (dict(n=17), dict(k=48), dict(n=8, gated=1), dict(n=1 << 17, gated=1), dict(k=1 << 18), dict(m=(1 << 17) + 1), dict(n=2 ** 31 - 16)):
        assert product(**bad) == UNSUPPORTED, bad
    for out in (1 << 24, (1 << 24) + 4 * 64 - 16, (1 << 24) - 4 * 32 + 16):        # rows of x, or of the result, in the other's
        assert product(m=4, out=C.c_void_p(out)) == INVALID
    need = lib.sp_fp4_product_workspace(64, 16, 8192, 0)                # columns cut, sums joined
    assert need > 0
    assert product(m=64, k=8192) == CAPACITY and product(m=64, k=8192, work=p[3], size=need - 1) == CAPACITY
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


# ---- the split of the attention's work (csrc/sp_plan.h, plain C++) ----
PLAN_DRIVER = r"""
#include <string.h>
#include "sp_plan.h"
extern "C" int split(int n, const int* rows, const int* spans, int n_q, int n_kv, int n_cu, long room, int* head, int* segs) {
  AttnPlan p;
  memset(&p, 0, sizeof(p));
  p.n_seg = n;
  for (int i = 0; i < n; ++i) { p.seg_rows[i] = rows[i]; p.seg_P[i] = spans[i] - rows[i]; p.seg_T[i] = rows[i]; }
  if (!attn_split_fp4(p, n_q, n_kv, n_cu, (size_t)room)) return 0;
  head[0] = p.qt; head[1] = p.total_items; head[2] = p.any_split; head[3] = p.units_total;
  for (int i = 0; i < n; ++i) {
    int* o = segs + 5 * i;
    o[0] = p.seg_item0[i]; o[1] = p.seg_chunks[i]; o[2] = p.seg_clen[i]; o[3] = p.seg_qblocks[i]; o[4] = p.seg_unit0[i];
  }
  return 1;
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan4")
    (d / "driver.cpp").write_text(PLAN_DRIVER)
    csrc = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2504_04104_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", csrc, str(d / "driver.cpp"), "-o", str(d / "driver.so")],
                   check=True)
    lib = C.CDLL(str(d / "driver.so"))

    def call(rows, spans, n_q=32, n_kv=8, n_cu=256, room=1 << 20):
        n = len(rows)
        head, segs = (C.c_int * 4)(), (C.c_int * (5 * n))()
        if not lib.split(n, (C.c_int * n)(*rows), (C.c_int * n)(*spans), n_q, n_kv, n_cu, C.c_long(room), head, segs):
            return None
        return list(head), np.array(segs).reshape(-1, 5)
    return call


def test_the_plan_covers_its_ranges(split):
    """Chunks are whole tiles and none is empty; the items and the partial rows of the requests follow each other; partial rows fit
    what there is for them; cut ranges make no more workgroups than there are CUs, give or take a request's rounding."""
    rng = np.random.default_rng(5)
    for _ in range(300):
        n = int(rng.integers(1, 65))
        rows = rng.integers(1, 257, n) if rng.random() < .3 else rng.integers(1, 9, n)
        spans = rows + rng.integers(0, 40000, n)
        n_q, n_kv = [(32, 8), (64, 8), (16, 4), (8, 8), (12, 2)][rng.integers(5)]
        room = int(rng.choice([0, 5000, 1 << 20]))
        (qt, items, any_split, units), segs = split(list(rows), list(spans), n_q, n_kv, 256, room)
        assert qt == 1 and units <= room
        g, item, unit = n_q // n_kv, 0, 0
        for i in range(n):
            item0, chunks, clen, qblocks, unit0 = segs[i]
            assert (item0, unit0, qblocks) == (item, unit, -(-rows[i] * g // 16))
            assert clen % 32 == 0 and (chunks - 1) * clen < spans[i] <= chunks * clen
            item += qblocks * chunks
            unit += chunks * rows[i] * n_q if chunks > 1 else 0
        assert (items, units, bool(any_split)) == (item, unit, max(s[1] for s in segs) > 1)
        assert not any_split or items * n_kv <= 256


def test_ranges_are_cut_where_it_pays(split):
    """One block of rows per head: from seven rounds of 256 slots saved; more blocks: from nine."""
    assert split([1], [1792])[0][2] == 0              # 7 rounds, one left of them in chunks
    assert split([1], [1793])[0][2] == 1
    assert split([16], [2560])[0][2] == 0             # four blocks, eight chunks: 10 rounds, two left of them, eight saved
    assert split([16], [2561])[0][2] == 1             # 11, nine saved
    assert split([16], [2304])[0][2] == 0             # 9 rounds; eight chunks of two: seven saved
    assert split([200], [40000])[0][2] == 0           # fifty blocks of eight heads: the CUs are full
    assert split([1] * 40, [40000] * 40)[0][2] == 0
    assert split([1], [40000], room=0)[0][2] == 0     # no room for partial rows
    assert split([1], [40000], room=5 * 32)[0][3] == 4 * 32
