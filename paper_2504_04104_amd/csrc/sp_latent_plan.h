// The split of a latent attention call's work, made on the host.  Plain C++.
#pragma once
#include "sp_plan.h"

#define LATENT_TILE 64             // slots that a workgroup takes at a time

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
    items += chunks * qblocks;
    if (chunks > 1) { units += (size_t)chunks * plan.seg_rows[i] * H; split = 1; }
  }
  plan.total_items = items;
  plan.units_total = (int)units;
  plan.any_split = split;
  plan.loads = ATTN_SHARED;
  return units;
}

inline bool latent_split(AttnPlan& plan, int H, int d_latent, int n_cu, size_t room) {
  int longest = 1;
  for (int i = 0; i < plan.n_seg; ++i) {
    const int tiles = (plan.seg_P[i] + plan.seg_T[i] + LATENT_TILE - 1) / LATENT_TILE;
    longest = tiles > longest ? tiles : longest;
  }
  double best = 1e30;
  int best_rows = 0, best_len = 0;
  for (int rows = 32; rows <= 64; rows += 32) {
    double work = 0.;
    for (int i = 0; i < plan.n_seg; ++i) {
      const long long qb = ((long long)plan.seg_rows[i] * H + rows - 1) / rows;
      work += (double)qb * ((plan.seg_P[i] + plan.seg_T[i] + LATENT_TILE - 1) / LATENT_TILE);
    }
    const double tile = rows == 32 ? 1.1 : 1.4;
    for (int cuts = 1; cuts <= longest; cuts = cuts < 4 ? cuts + 1 : cuts + cuts / 3) {
      const int len = (longest + cuts - 1) / cuts;
      long long items = 0;
      double units = 0.;
      for (int i = 0; i < plan.n_seg; ++i) {
        const int tiles = (plan.seg_P[i] + plan.seg_T[i] + LATENT_TILE - 1) / LATENT_TILE, chunks = (tiles + len - 1) / len;
        items += ((long long)plan.seg_rows[i] * H + rows - 1) / rows * chunks;
        if (chunks > 1) units += (double)chunks * plan.seg_rows[i] * H;
      }
      if (units > (double)room && cuts > 1) break;
      const double rounds = (double)items / n_cu;
      double t = rounds <= 1. ? len : work / n_cu + 0.5 * len;
      if (t < len) t = len;
      t = t * tile + 2. * (rounds <= 1. ? 1. : rounds);
      if (units > 0.) t += 5. + units * d_latent * 8. / 4e6;
      if (t < best) { best = t; best_rows = rows; best_len = len; }
    }
  }
  const size_t units = latent_cut(plan, H, best_rows, best_len);
  return units <= room;
}
