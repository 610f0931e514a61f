"""The split of a latent attention call's work (csrc/sp_latent_plan.h, plain C++) on the CPU."""
import ctypes as C
import os
import random
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_04104_amd", "csrc")
DRIVER = """
#include <string.h>
#include "sp_latent_plan.h"
extern "C" int split(int n, const int* rows, const int* spans, int heads, int d_latent, int n_cu, long room, int* head, int* segs) {
  AttnPlan p;
  memset(&p, 0, sizeof(p));
  p.n_seg = n;
  for (int i = 0; i < n; ++i) { p.seg_rows[i] = rows[i]; p.seg_T[i] = rows[i] < spans[i] ? rows[i] : spans[i]; p.seg_P[i] = spans[i] - p.seg_T[i]; }
  if (!latent_split(p, heads, d_latent, n_cu, (size_t)room)) return 0;
  const int h[] = {p.qt, p.total_items, p.any_split, p.units_total};
  memcpy(head, h, sizeof(h));
  for (int i = 0; i < n; ++i) {
    const int s[] = {p.seg_item0[i], p.seg_chunks[i], p.seg_clen[i], p.seg_qblocks[i], p.seg_unit0[i]};
    memcpy(segs + i * 5, s, sizeof(s));
  }
  return 1;
}
extern "C" void item(int local, int blocks, int chunks, int* block, int* chunk) {
  const LatentItem w = latent_item(local, blocks, chunks);
  *block = w.block; *chunk = w.chunk;
}
extern "C" int items(int blocks, int chunks) { return latent_items(blocks, chunks); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "driver.cpp").write_text(DRIVER)
    so = str(d / "driver.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "driver.cpp"), "-o", so], check=True)
    return C.CDLL(so)


def split(lib, rows, spans, heads, d_latent=512, n_cu=256, room=40960):
    r, s = ((C.c_int * len(rows))(*v) for v in (rows, spans))
    head, segs = (C.c_int * 4)(), (C.c_int * (5 * len(rows)))()
    if not lib.split(len(rows), r, s, heads, d_latent, n_cu, C.c_long(room), head, segs):
        return None
    out = dict(zip(("qt", "items", "any_split", "units"), head))
    out["segs"] = np.array(segs).reshape(-1, 5).tolist()
    return out


def test_every_plan_covers_its_ranges(lib):
    """Chunks are whole tiles, none is empty, they cover the range; blocks cover the query rows; items and partial rows of the requests
    follow each other; the partial rows fit the room, and no call is refused (a chunk each needs none)."""
    r = random.Random(2)
    for _ in range(3000):
        heads = r.choice([1, 3, 8, 16, 64, 128, 1024])
        rows = [r.choice([1, 2, 5, 17, 64, 256]) for _ in range(r.choice([1, 1, 2, 5, 31, 64]))]
        spans = [v + int(2 ** r.uniform(0, r.choice([8, 15, 20]))) for v in rows]
        room = r.choice([0, 2000, 40960])
        p = split(lib, rows, spans, heads, r.choice([256, 512]), r.choice([32, 256]), room)
        assert p["qt"] in (2, 4)
        item, unit, any_split = 0, 0, 0
        for (item0, chunks, clen, qblocks, unit0), m, span in zip(p["segs"], rows, spans):
            assert clen % 64 == 0 and (chunks - 1) * clen < span <= chunks * clen
            assert qblocks == -(-m * heads // (16 * p["qt"]))
            assert (item0, unit0) == (item, unit)
            item += lib.items(qblocks, chunks)
            unit += chunks * m * heads if chunks > 1 else 0
            any_split |= chunks > 1
        assert (item, unit, any_split) == (p["items"], p["units"], p["any_split"])
        assert unit <= room


def test_every_block_and_chunk_has_one_workgroup(lib):
    """Workgroups without a chunk are fewer than eight a block; a chunk's workgroups go to one XCD (the same number modulo eight) where
    there are eight chunks and more."""
    b, c = C.c_int(), C.c_int()
    for blocks in (1, 2, 3, 5, 16, 31):
        for chunks in (1, 2, 7, 8, 9, 15, 16, 17, 63, 64, 100):
            n = lib.items(blocks, chunks)
            assert n < (chunks + 8) * blocks
            seen, xcd = set(), {}
            for i in range(n):
                lib.item(i, blocks, chunks, C.byref(b), C.byref(c))
                assert 0 <= b.value < blocks and c.value >= 0
                if c.value >= chunks:
                    continue
                assert (b.value, c.value) not in seen
                seen.add((b.value, c.value))
                if chunks >= 8:
                    assert xcd.setdefault(c.value, i % 8) == i % 8
            assert len(seen) == blocks * chunks


def test_one_row_of_a_short_range_is_not_split(lib):
    assert split(lib, [1], [1], 16)["any_split"] == 0
    assert split(lib, [1] * 64, [64] * 64, 16)["any_split"] == 0


def test_few_rows_of_a_long_range_fill_the_card(lib):
    p = split(lib, [5], [32768], 16)
    assert 128 <= p["items"] <= 256
