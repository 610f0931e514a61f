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
extern "C" void unpack(int v, int* group, int* groups, int* start) { const LatentPlace p = latent_unpack(v); *group = p.group; *groups = p.groups; *start = p.start; }
extern "C" int first_of(int start, int x) { return latent_first(start, x); }
extern "C" int units_on(int units, int start, int x) { return latent_units_on(units, start, x); }
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


def placed(lib, v):
    group, groups, start = C.c_int(), C.c_int(), C.c_int()
    lib.unpack(v, C.byref(group), C.byref(groups), C.byref(start))
    return group.value, groups.value, start.value


def workgroups(lib, p):
    """(request, block, chunk) of every workgroup, None for those without, found as the kernel finds them."""
    segs = []
    for v, chunks, _, blocks, _ in p["segs"]:
        group, groups, start = placed(lib, v)
        assert groups == -(-blocks // group) and 0 <= start < 8
        segs.append((group, start, groups, chunks, blocks))
    out = []
    for i in range(p["items"]):
        x, local, work = i % 8, i // 8, None
        for seg, (group, start, groups, chunks, blocks) in enumerate(segs):
            n = lib.units_on(chunks * groups, start, x) * group
            if local < n:
                unit = lib.first_of(start, x) + local // group * 8
                chunk, block = unit // groups, unit % groups + local % group * groups
                assert chunk < chunks
                work = (seg, block, chunk) if block < blocks else None
                break
            local -= n
        out.append(work)
    return out


def random_calls(n, seed):
    r = random.Random(seed)
    for _ in range(n):
        heads = r.choice([1, 3, 8, 16, 64, 128, 1024])
        rows = [r.choice([1, 2, 5, 17, 64, 256]) for _ in range(r.choice([1, 1, 2, 5, 31, 64]))]
        spans = [v + int(2 ** r.uniform(0, r.choice([8, 15, 20]))) for v in rows]
        yield rows, spans, heads, r.choice([256, 512]), r.choice([32, 256]), r.choice([0, 2000, 40960])


def test_every_plan_covers_its_ranges(lib):
    """Chunks are whole tiles, none is empty, they cover the range; blocks cover the query rows; the requests' partial rows follow each
    other; they fit the room, and no call is refused (a chunk each needs none)."""
    for rows, spans, heads, d_latent, n_cu, room in random_calls(2000, 2):
        p = split(lib, rows, spans, heads, d_latent, n_cu, room)
        assert p["qt"] in (2, 4)
        unit, any_split = 0, 0
        for (_, chunks, clen, qblocks, unit0), m, span in zip(p["segs"], rows, spans):
            assert clen % 64 == 0 and (chunks - 1) * clen < span <= chunks * clen
            assert qblocks == -(-m * heads // (16 * p["qt"]))
            assert unit0 == unit
            unit += chunks * m * heads if chunks > 1 else 0
            any_split |= chunks > 1
        assert (unit, any_split) == (p["units"], p["any_split"])
        assert unit <= room


def test_every_block_and_chunk_has_one_workgroup(lib):
    """Also: what an XCD has is at most an eighth more than its share, one workgroup a CU where a share is that; groups of a chunk stay on one XCD."""
    for rows, spans, heads, d_latent, n_cu, room in random_calls(300, 3):
        p = split(lib, rows, spans, min(heads, 128), d_latent, n_cu, room)
        if p["items"] > 30000:
            continue
        work = workgroups(lib, p)
        real = [w for w in work if w is not None]
        assert len(set(real)) == len(real) == sum(chunks * blocks for _, chunks, _, blocks, _ in p["segs"])
        share = -(-len(real) // 8)
        longest = -(-len(work) // 8)
        assert longest <= share + max(1, share // 8)
        assert longest <= n_cu // 8 or share > n_cu // 8
        where = {}
        for i, w in enumerate(work):
            if w is not None:
                seg, block, chunk = w
                where.setdefault((seg, chunk, block % placed(lib, p["segs"][seg][0])[1]), set()).add(i % 8)
        assert all(len(v) == 1 for v in where.values())


def test_blocks_of_a_chunk_go_together_where_there_is_enough_else(lib):
    """32 requests with two blocks each in five chunks: every chunk's blocks on one XCD.  Ranges that stay in L2: one by one."""
    p = split(lib, [8] * 32, [2600] * 32, 16)
    assert all(placed(lib, v)[0] == blocks for v, _, _, blocks, _ in p["segs"])
    for rows, spans, heads in (([128], [4224], 64), ([2] * 8, [900] * 8, 128)):
        p = split(lib, rows, spans, heads)
        assert all(placed(lib, v)[0] == 1 for v, *_ in p["segs"])
        assert p["items"] == sum(chunks * blocks for _, chunks, _, blocks, _ in p["segs"])


def test_one_row_of_a_short_range_is_not_split(lib):
    assert split(lib, [1], [1], 16)["any_split"] == 0
    assert split(lib, [1] * 64, [64] * 64, 16)["any_split"] == 0


def test_few_rows_of_a_long_range_fill_the_card(lib):
    p = split(lib, [5], [32768], 16)
    assert 128 <= p["items"] <= 256
