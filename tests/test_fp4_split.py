"""How products with 4-bit weights are cut (csrc/sp_fp4_split.h, plain C++), and that the GPU tests' cases reach every kernel."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2504_04104_amd as sp
from fp4_cases import FORWARDS, PRODUCTS

DRIVER = r"""
#include "sp_fp4_split.h"
extern "C" void cut(int kind, int m, int n, int k, int n_cu, long room, int* o) {
  const Fp4Split f = kind == 0 ? fp4_split_call(m, n, k, n_cu) : kind == 1 ? fp4_split_parts(m, n, k, n_cu, (size_t)room)
                                                                           : fp4_split_gateup(m, n, k, n_cu);
  o[0] = f.mt; o[1] = f.ns; o[2] = f.S;
}
extern "C" int parts_free(int m, int n, int k, int n_cu, int* o) {
  const Fp4Split f = fp4_split(m, n, k, n_cu, 0.f, FP4_MOST_SLICES);
  o[0] = f.mt; o[1] = f.ns; o[2] = f.S;
  return f.mt ? 0 : 1;
}
extern "C" long bytes(int n, int k) { return (long)fp4_bytes(n, k); }
"""
CALL, PARTS, GATEUP = 0, 1, 2
TILED = [(1, 2), (2, 2), (4, 2), (4, 4), (5, 4), (7, 4)]
FEW = [(0, 1), (0, 2), (0, 4)]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("split4")
    (d / "driver.cpp").write_text(DRIVER)
    csrc = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2504_04104_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", csrc, str(d / "driver.cpp"), "-o", str(d / "driver.so")], check=True)
    out = C.CDLL(str(d / "driver.so"))
    out.bytes.restype = C.c_long
    return out


def cut(lib, kind, m, n, k, n_cu=256, room=1 << 40):
    o = (C.c_int * 3)()
    lib.cut(kind, m, n, k, n_cu, C.c_long(room), o)
    return tuple(o)


def steps(k, S, mt):
    """Steps of the loop over the chunks of 128 columns, of the longest slice: in turns of four, the rest behind the loop."""
    units, groups = -(-k // 256), 2 if mt <= 2 else 1
    return max(-(-(min((s + 1) * units // S * 2, -(-k // 128)) - s * units // S * 2) // groups) for s in range(S))


def turns(k, S, mt):
    """More than two turns of the loop and steps behind it: what a short product, or one that ends with a turn, leaves out."""
    return steps(k, S, mt) >= 9 and steps(k, S, mt) % 4 != 0


def test_cuts_are_within_their_bounds(lib):
    rng = np.random.default_rng(2)
    for _ in range(4000):
        m, n, k = (int(2 ** rng.uniform(0, 17)), 16 * int(2 ** rng.uniform(0, 13)), 32 * int(2 ** rng.uniform(0, 12)))
        n_cu, room = int(rng.choice([32, 64, 128, 256])), int(2 ** rng.uniform(10, 34))
        assert lib.bytes(n, k) == sp.load_library().sp_fp4_matrix_bytes(n, k)
        for kind in (CALL, PARTS, GATEUP):
            mt, ns, S = cut(lib, kind, m, n if kind != GATEUP else max(16, n // 2), k, n_cu, room)
            assert (mt, ns) in TILED + FEW
            assert mt > 0 or (m <= 16 and S <= 1)
            assert S <= 16 and S <= -(-k // 256) and (kind != GATEUP or S == 1)
            assert S >= (0 if kind == PARTS else 1) and (kind != PARTS or S * m * n <= room)
            assert kind != PARTS or S >= 1 or m * n > room


def test_products_reach_every_kernel_and_its_loop(lib):
    seen = set()
    for m, n, k, gated in PRODUCTS:
        assert k % 32 == 0 and n % 16 == 0
        mt, ns, S = cut(lib, CALL, m, n * 2 if gated else n, k)
        if mt == 0 or turns(k, S, mt):
            seen.add((mt, ns, S > 1, gated))
    want = {(mt, ns, cut_, gated) for mt, ns in TILED for cut_ in (False, True) for gated in (False, True)}
    want |= {(mt, ns, False, gated) for mt, ns in FEW for gated in (False, True)}
    assert seen == want


def forward_cuts(lib, d, nq, nkv, ff, m):
    """(what, tiles, strips, rows in fragment order, loop) of the four products of a layer."""
    dq, nqkv, rows = nq * 128, (nq + 2 * nkv) * 128, -(-m // 16) * 16
    room = max(max(rows, 1024) * max(nqkv, d), rows * 2 * ff)
    for what, n, k in (("parts", nqkv, d), ("parts", d, dq), ("parts", d, ff), ("gated", ff, d)):
        mt, ns, S = cut(lib, PARTS if what == "parts" else GATEUP, m, n, k, room=room)
        yield what, mt, ns, m > 8, mt == 0 or turns(k, S, mt)


def test_forward_calls_reach_every_kernel_and_its_loop(lib):
    seen = set()
    for case in FORWARDS:
        seen |= set(forward_cuts(lib, *case))
    want = {("gated", mt, ns, m > 8, True) for mt, ns in FEW for m in (8, 9)} | {(what, 1, 2, False, True) for what in ("parts", "gated")}
    want |= {(what, mt, ns, True, True) for mt, ns in TILED for what in ("parts", "gated")}
    want.add(("parts", 0, 4, False, True))          # one or two rows of more than 32768 columns
    assert want <= seen


def test_partial_sums_have_the_kernel_for_few_rows_where_it_is_the_faster_one(lib):
    """The kernels that partial sums do not have would be chosen nowhere: the cut is what it is with all of them."""
    rng = np.random.default_rng(4)
    n_few, free = 0, (C.c_int * 3)()
    for i in range(20000):
        m, units = int(rng.integers(1, 17 if i % 2 else 3)), int(2 ** rng.uniform(0, 9))
        strips = int(rng.integers(2000, 3200)) if i % 4 == 0 else int(2 ** rng.uniform(0, 13))
        n_cu = int(rng.choice([32, 64, 128, 256]))
        n_few += lib.parts_free(m, strips * 16, units * 256, n_cu, free)
        assert cut(lib, PARTS, m, strips * 16, units * 256, n_cu) == tuple(free), (m, units, strips, n_cu)
    assert n_few > 100


PLAN_DRIVER = r"""
#include <string.h>
#include "sp_plan.h"
extern "C" int chunks(int n, const int* rows, const int* spans, int n_q, int n_kv, long room) {
  AttnPlan p;
  memset(&p, 0, sizeof(p));
  p.n_seg = n;
  for (int i = 0; i < n; ++i) { p.seg_rows[i] = rows[i]; p.seg_P[i] = spans[i] - rows[i]; p.seg_T[i] = rows[i]; }
  return attn_split_fp4(p, n_q, n_kv, 256, (size_t)room) ? p.any_split : -1;
}
"""


def test_calls_that_are_to_be_cut_are(tmp_path):
    from test_gpu_fp4_calls import CALLS, KINDS, KV, REPLAYED
    (tmp_path / "driver.cpp").write_text(PLAN_DRIVER)
    csrc = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2504_04104_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", csrc, str(tmp_path / "driver.cpp"), "-o", str(tmp_path / "driver.so")], check=True)
    plan = C.CDLL(str(tmp_path / "driver.so"))

    def is_cut(rows, spans, nq=8, nkv=2, most=64):
        rows, spans = zip(*sorted(zip(rows, spans), key=lambda p: -p[1]))
        n = len(rows)
        return plan.chunks(n, (C.c_int * n)(*rows), (C.c_int * n)(*spans), nq, nkv, C.c_long(most * nq * 32))
    for sh, flags, _, _ in KINDS.values():
        for name, reqs in CALLS.items():
            if flags & KV:
                assert is_cut([n for *_, n in reqs], [sum(r) for r in reqs], sh.n_q_heads, sh.n_kv_heads, 256) == name.startswith("cut")
    for name, (flags, _, _, rows, contexts) in REPLAYED.items():
        if flags & KV:                              # whatever request has which context
            for turn in range(len(rows)):
                spans = [contexts[(i + turn) % len(rows)] + max(rows) + 3 for i in range(len(rows))]
                assert is_cut(rows, spans) == name.endswith("_cut")
    assert is_cut([4], [6004], 32, 8) and is_cut([5], [7005], 32, 8)  # two captured graphs of one stage
