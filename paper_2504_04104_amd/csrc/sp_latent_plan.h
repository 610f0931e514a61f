// The split of a latent attention call's work, made on the host.  Plain C++.
#pragma once
#include "sp_plan.h"

#define LATENT_TILE 64             // slots that a workgroup takes at a time

// Workgroups of a request, (block of query rows, chunk) by number: chunk after chunk for every block, or, where there are eight chunks and
// more, eight chunks side by side for every block, so that a chunk's blocks run on the XCD whose L2 has it (consecutive workgroups go
// round over the eight; 80 rows behind 32749 slots in 64 chunks 24.7 us, in 74, which scattered them, 30.3).  The last eight chunks
// may be part empty: chunk >= chunks then, nothing to do.
struct LatentItem { int block, chunk; };
#ifdef __HIPCC__
__host__ __device__
#endif
inline LatentItem latent_item(int local, int blocks, int chunks) {
  if (chunks < 8 || blocks == 1) return {local / chunks, local % chunks};
  const int eights = local >> 3;
  return {eights % blocks, eights / blocks * 8 + (local & 7)};
}
inline int latent_items(int blocks, int chunks) { return (chunks < 8 || blocks == 1 ? chunks : (chunks + 7) / 8 * 8) * blocks; }

// Every request's range in chunks of at most `len` tiles, blocks of `rows` query rows; returns the partial rows that this takes.
inline size_t latent_cut(AttnPlan& plan, int H, int rows, int len) {
  size_t units = 0;
  int items = 0, split = 0;
  plan.qt = rows / 16;
  for (int i = 0; i < plan.n_seg; ++i) {
    const int span = plan.seg_P[i] + plan.seg_T[i], tiles = (span + LATENT_TILE - 1) / LATENT_TILE;
    const int want = (tiles + len - 1) / len, each = (tiles + want - 1) / want, chunks = (tiles + each - 1) / each;
    const int qblocks = (int)(((long long)plan.seg_rows[i] * H + rows - 1) / rows);
    plan.seg_item0[i] = items; plan.seg_chunks[i] = chunks; plan.seg_clen[i] = each * LATENT_TILE; plan.seg_qblocks[i] = qblocks;
    plan.seg_unit0[i] = (int)units;
    items += latent_items(qblocks, chunks);
    if (chunks > 1) { units += (size_t)chunks * plan.seg_rows[i] * H; split = 1; }
  }
  plan.total_items = items;
  plan.units_total = (int)units;
  plan.any_split = split;
  plan.loads = ATTN_SHARED;
  return units;
}

// Blocks of 32 or 64 query rows and chunks of the ranges, by the time that they would take: a tile of 64 slots is 1.3 us of a workgroup of
// 32 rows and 1.75 of one of 64 (d_latent 512; what LDS gives a clock bounds both), a workgroup has 4.5 us beside its tiles, a CU
// room for one; chunks cost the merge, a launch and the partial rows on their way out and back.  Both sides, us a call, best cut of each:
// 16 rows behind 512 slots 12.7 in blocks of 32 and 13.3 of 64; 80 behind 32749 24.8 and 25.9; 2048 behind 2048 29.5 and 28.1; 32
// requests' 16 to 128 behind 512 to 4096 42.5 and 35.9; 8192 behind 4096 90.4 (a chunk) and 79.1 (two).  What is picked is within 8 % of the
// best of all cuts there.  False: the partial rows do not fit.
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
  return latent_cut(plan, H, best_rows, best_len) <= room;
}
