// The split of a latent attention call's work, made on the host.  Plain C++.
#pragma once
#include "sp_plan.h"

#define LATENT_TILE 64             // slots that ranges are cut at multiples of: two of the tiles that a workgroup takes at a time
#define LATENT_FAR (16 << 20)      // bytes of latents that a call reads from where they do not stay in L2

// Workgroups of a call.  Consecutive ones go round over the eight XCDs: workgroup i is number i / 8 of those of XCD i % 8.  A request's work is
// cut into units, a chunk and `group` of its blocks of query rows, every groups-th from one on (some may be short: workgroups without a
// block), which follow each other over the XCDs from `start` on, request after request: the blocks of a unit read the same rows at the same
// time behind the same L2.
struct LatentPlace { int group, groups, start; };           // (blocks are at most 8192: 256 nodes x 1024 heads in blocks of 32)
#ifdef __HIPCC__
#define LATENT_BOTH __host__ __device__
#else
#define LATENT_BOTH
#endif
inline int latent_pack(LatentPlace p) { return p.groups << 17 | p.group << 3 | p.start; }
LATENT_BOTH inline LatentPlace latent_unpack(int v) { return {(v >> 3) & 0x3fff, v >> 17, v & 7}; }
// The request's first unit on XCD x, and how many it has there.
LATENT_BOTH inline int latent_first(int start, int x) { return (x - start) & 7; }
LATENT_BOTH inline int latent_units_on(int units, int start, int x) {
  const int j = latent_first(start, x);
  return j < units ? ((units - 1 - j) >> 3) + 1 : 0;
}

// Groups of up to `most` blocks; returns the longest row of workgroups of an XCD.
inline int latent_place(AttnPlan& plan, int most) {
  int load[8] = {0, 0, 0, 0, 0, 0, 0, 0}, start = 0, longest = 0, grid = 0;
  for (int i = 0; i < plan.n_seg; ++i) {
    const int blocks = plan.seg_qblocks[i], cut = (blocks + most - 1) / most, group = (blocks + cut - 1) / cut, groups = (blocks + group - 1) / group;
    const int units = plan.seg_chunks[i] * groups;
    plan.seg_item0[i] = latent_pack({group, groups, start});
    for (int x = 0; x < 8; ++x) load[x] += latent_units_on(units, start, x) * group;
    start = (start + units) & 7;
  }
  for (int x = 0; x < 8; ++x) {
    longest = load[x] > longest ? load[x] : longest;
    if (load[x] > 0 && (load[x] - 1) * 8 + x + 1 > grid) grid = (load[x] - 1) * 8 + x + 1;
  }
  plan.total_items = grid;
  return longest;
}
// Groups of up to four blocks where the rows that the call reads are too many for the L2s, 4 MB each, to have a chunk when it is asked for
// again, and the XCDs stay nearly level (us a call on one set of rows over and over: 32 requests of 1 to 8 nodes x 16 heads, 75 MB, 33.2, one
// by one 36.6; 80 query rows behind 32749 slots 26.5 and 29.9); else one by one (64 nodes x 32 heads behind 2048, 2 MB: 28.1, in groups of 32
// 30.0; 8 requests of 1 to 2 nodes x 128 heads, 6 MB: in blocks of 64 22.5, in groups 24.2, in the blocks of 32 that the rule below
// takes 21.2 and 22.3, where an order that asks for no XCD took 19.8: the one case measured that this placement costs).  Pairs are of one
// run; between runs and cards a call moves by up to a tenth.
inline void latent_place(AttnPlan& plan, long long items, int n_cu, long long bytes) {
  int most = 1;
  if (bytes > LATENT_FAR)
    for (int i = 0; i < plan.n_seg; ++i) most = plan.seg_qblocks[i] > most ? plan.seg_qblocks[i] : most;
  if (most > 4) most = 4;
  const long long share = (items + 7) / 8, per = n_cu / 8;
  long long allowed = share + (share < 8 ? 1 : share / 8);
  if (share <= per && allowed > per) allowed = per;
  while (latent_place(plan, most) > allowed && most > 1) --most;
}

// Every request's range in chunks of at most `len` tiles, blocks of `rows` query rows; returns the partial rows that this takes.
inline size_t latent_cut(AttnPlan& plan, int H, int d_latent, int rows, int len, int n_cu) {
  size_t units = 0;
  long long items = 0, slots = 0;
  int split = 0;
  plan.qt = rows / 16;
  for (int i = 0; i < plan.n_seg; ++i) {
    const int span = plan.seg_P[i] + plan.seg_T[i], tiles = (span + LATENT_TILE - 1) / LATENT_TILE;
    const int want = (tiles + len - 1) / len, each = (tiles + want - 1) / want, chunks = (tiles + each - 1) / each;
    const int qblocks = (int)(((long long)plan.seg_rows[i] * H + rows - 1) / rows);
    plan.seg_chunks[i] = chunks; plan.seg_clen[i] = each * LATENT_TILE; plan.seg_qblocks[i] = qblocks;
    plan.seg_unit0[i] = (int)units;
    items += (long long)qblocks * chunks;
    slots += span;
    if (chunks > 1) { units += (size_t)chunks * plan.seg_rows[i] * H; split = 1; }
  }
  plan.units_total = (int)units;
  plan.any_split = split;
  plan.loads = ATTN_SHARED;
  latent_place(plan, items, n_cu, slots * d_latent * 2);
  return units;
}

// Blocks of 32 or 64 query rows and chunks of the ranges, by the time that they would take: 64 slots are 1.3 us of a workgroup of 32 rows
// and 1.75 of one of 64 (d_latent 512; what LDS gives a clock bounds blocks of 64, and not those of 32: half of their scores' LDS reads left
// out, for timing, took 5 % off), a workgroup has 4.5 us beside its tiles, a CU room for one; chunks cost the merge, a launch and the
// partial rows on their way out and back.  Both sides, us a call, best cut of each:
// 16 rows behind 512 slots 12.7 in blocks of 32 and 13.3 of 64; 80 behind 32749 24.8 and 25.9; 2048 behind 2048 29.5 and 28.1; 32
// requests' 16 to 128 behind 512 to 4096 42.5 and 35.9; 8192 behind 4096 90.4 (a chunk) and 79.1 (two).  What is picked is within 8 % of the
// best of all cuts there.  At d_latent 256 a tile is taken for 0.575 of 512's, which was not fitted by itself: what is picked is within 7 %
// of the best cut (16 rows behind 512 10.8 in blocks of 32 and 11.1 of 64; 80 behind 32749 18.6 and 20.3; 2048 behind 2048 18.4 and 18.6;
// 1280 each of 4 requests behind 2000 to 4000 38.8 and 34.4; 8192 behind 4096 58.0 and 50.4).  Rounds are not counted whole: a call of
// little more than one, or whose partial rows would not fit, is cut less than would be best.  False: the partial rows do not fit.
inline bool latent_split(AttnPlan& plan, int H, int d_latent, int n_cu, size_t room) {
  int tiles[SP_BATCH], longest = 1;
  for (int i = 0; i < plan.n_seg; ++i) {
    tiles[i] = (plan.seg_P[i] + plan.seg_T[i] + LATENT_TILE - 1) / LATENT_TILE;
    longest = tiles[i] > longest ? tiles[i] : longest;
  }
  double best = 1e30;
  int best_rows = 64, best_len = longest;
  for (int rows = 32; rows <= 64; rows += 32) {
    int blocks[SP_BATCH];
    double work = 0.;
    for (int i = 0; i < plan.n_seg; ++i) {
      blocks[i] = (int)(((long long)plan.seg_rows[i] * H + rows - 1) / rows);
      work += (double)blocks[i] * tiles[i];
    }
    const double tile = (rows == 32 ? 1.3 : 1.75) * (0.15 + 0.85 / 512. * d_latent);
    for (int cuts = 1, len = longest, before = 0; cuts <= longest; cuts = cuts < 8 ? cuts + 1 : cuts + cuts / 4) {
      len = (longest + cuts - 1) / cuts;
      if (len == before) continue;
      before = len;
      long long items = 0, units = 0;
      for (int i = 0; i < plan.n_seg; ++i) {
        const int chunks = tiles[i] <= len ? 1 : (tiles[i] + len - 1) / len;
        items += (long long)blocks[i] * chunks;
        if (chunks > 1) units += (long long)chunks * plan.seg_rows[i] * H;
      }
      if (units > (long long)room) break;
      const double rounds = (double)items / n_cu;
      double t = rounds <= 1. ? len : work / n_cu + 0.5 * len;
      if (t < len) t = len;
      t = t * tile + 4.5 * (rounds <= 1. ? 1. : rounds);
      if (units > 0) t += 4.5 + (double)units * d_latent * 8. / 4.5e6;
      if (t < best) { best = t; best_rows = rows; best_len = len; }
      if (rounds > 4.) break;                      // (shorter chunks: more of everything but the last one's time)
    }
  }
  return latent_cut(plan, H, d_latent, best_rows, best_len, n_cu) <= room;
}
