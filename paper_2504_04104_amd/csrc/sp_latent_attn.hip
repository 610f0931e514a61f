// Tree attention over a latent cache on the matrix cores: d_latent 256 and 512, d_rope 32 and 64.
//
//   out = softmax(scale * q . [c | r]) c     over the rows [c | r] of the cache that the node sees (committed context, ancestors, itself)
//
// The cache has one row a slot for all heads, so the nodes and heads of a request are the rows of one matrix, node * heads + head, and
// a workgroup takes 32 or 64 of them along a chunk of the request's range: 2 (2 d_latent + d_rope) operations a row and slot stand
// against the slot's (d_latent + d_rope) * 2 bytes.  Tiles of 32 slots lie in LDS as they lie in the cache and are used from there twice:
// rows of them for the scores (16x16x32), columns of them, by the transposing reads, for the results (32x32x16).  The 64 x 512 float32
// results fill the registers of four waves; the other four form the scores, weights and row sums, a tile ahead, so that every SIMD has a
// wave of either kind and one's products pass behind the other's LDS reads and exponentials (eight waves that did both in turn: 118 us a
// call, this way 93).  Four tiles are in LDS: two on their way, one under the scores, one under the results; one barrier a tile.
//
// Running softmax with a shift that hardly ever moves: a row's weights are exp2 of its score less a past maximum, and only where a tile
// has weights past 2^16 are its maxima taken, the row's results scaled, and the tile taken again.  Weights are rounded to bf16 (2^-8 of
// each at most), and the row's sum is that of the rounded ones, so that what rounding adds to numerator and denominator is the same; all
// else is float32.  Chunks leave unnormalized results, sums and shifts, which k_latent_merge_few and k_latent_merge join.
//
// Bound by LDS and the clock under full load (1.75 to 1.83 of 2.4 GHz): a tile of 64 rows takes 1736 cycles where its reads (scores 576 and 160,
// results 256) and the rows coming in (288) need 1280 at 128 bytes a clock and its products 1088.  A workgroup has 4.5 us beside its
// tiles (first rows, query rows, results out).  512 + 64 columns: 128 nodes x 64 heads behind 4096 slots 71 to 76 us, 1.05 PFLOP/s (a large
// library product 1.41), and 8.8 of merge; 64 x 32 behind 2048 22 and 5.2; 16 rows behind 512
// 9.3 and 3.9; 256 x 128 behind 4096, one chunk, 262 to 272, 1.16 PFLOP/s.  256 + 32: 51 and 6.1, 15.7 and 4.1, 7.0 and 3.3.
#include "sp_latent_plan.h"
#include "sp_launch.h"

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;

// Sixteen lanes read 8 bytes each; lane 4c + x of them gets element x of what lanes c, 4 + c, 8 + c and 12 + c read.
__device__ __forceinline__ uint2 read_transposed(const char* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p)));
#else
  return uint2{0u, 0u};
#endif
}
__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// acc + the two halves of w
__device__ __forceinline__ float dot2(uint32_t w, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), acc, false);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Sums over the lanes up to one's own.
__device__ __forceinline__ int wave_scan(int v) {
#ifdef __HIP_DEVICE_COMPILE__
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);         // from 1, 2, 4 and 8 lanes below in rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);         // a row's last lane to the second and fourth
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);         // the second row's to the upper half
#endif
  return v;
}

#define LW 8                       // waves per workgroup: four form scores, four the results
#define LK 32                      // slots per tile

// Places of 16-byte units in LDS: rows of 256 bytes, of 128 and of 64.  Sixteen rows' units of the same columns lie in sixteen
// different places.
__device__ __forceinline__ int swap256(int row) { return (row & 3) * 4 + ((row >> 2) & 3); }
__device__ __forceinline__ int swap128(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swap64(int row) { return (row >> 2) & 3; }

// R query rows (32 or 64) per workgroup.
template <int DC, int DR, int R, bool PAGED>
__global__ void __launch_bounds__(64 * LW, 2) k_latent_attn(LatentAttnArgs a, AttnPlan plan) {
  constexpr int SUB = DC / 128, ROW = (DC + DR) * 2, KR = DR / 32, NS = DC / 32 + KR;
  constexpr int SUB_B = LK * 256, TILE = SUB * SUB_B + LK * DR * 2;
  constexpr int CG = DC / 256, RT = R / 32;        // results: CG x 64 columns, RT x 32 rows a wave
  constexpr int TQ = R / 32;                       // scores: TQ x 16 rows a wave
  constexpr bool STAGED = R == 64;                 // query rows by way of LDS
  __shared__ __attribute__((aligned(16))) char s_0[TILE], s_1[TILE], s_2[TILE], s_3[TILE];
  __shared__ __attribute__((aligned(16))) char s_p[2][R * LK * 2];
  __shared__ __attribute__((aligned(16))) float s_max[R][2];
  __shared__ uint32_t s_anc[R][12];                // ancestor masks of the query rows, a word of zeros in front, three behind
  __shared__ int s_redo;

  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, kg = lane >> 4;
  const int xcd = blockIdx.x & 7;
  int seg = 0, local = blockIdx.x >> 3;            // the workgroup's request, and its number among the request's on this XCD
  if (plan.n_seg > 1) {
    int n = 0;
    if (lane < plan.n_seg) {
      const LatentPlace p = latent_unpack(plan.seg_item0[lane]);
      n = latent_units_on(plan.seg_chunks[lane] * p.groups, p.start, xcd) * p.group;
    }
    const int to = wave_scan(n);                   // workgroups of the requests up to the lane's
    seg = uni(__popcll(__builtin_amdgcn_ballot_w64(lane < plan.n_seg && to <= local)));
    if (seg >= plan.n_seg) return;
    local -= __builtin_amdgcn_readlane(to - n, seg);
  }
  const LatentPlace place = latent_unpack(plan.seg_item0[seg]);
  // (quotients of numbers below 2^21 by way of float32: half a step of the quotient is more than they are off)
  const int group = place.group, groups = place.groups, nth = uni((int)(((float)local + 0.5f) * __builtin_amdgcn_rcpf((float)group)));
  const int unit = latent_first(place.start, xcd) + nth * 8;
  const int chunks = plan.seg_chunks[seg], seg_rows = plan.seg_rows[seg], row0 = plan.seg_row0[seg], req = plan.seg_req[seg];
  const int P = plan.seg_P[seg], span = P + plan.seg_T[seg], clen = plan.seg_clen[seg];
  const int ch = uni((int)(((float)unit + 0.5f) * __builtin_amdgcn_rcpf((float)groups))), qb = unit - ch * groups + (local - nth * group) * groups;
  if (ch >= chunks || qb >= plan.seg_qblocks[seg]) return;
  const int H = a.d.n_heads, nq = seg_rows * H;    // query rows of the request, node * H + head
  const int c0 = ch * clen, c1 = min(c0 + clen, span), tiles = (c1 - c0 + LK - 1) / LK;

  // Rows of the cache, and the query rows first: a wave brings eight of them, whole lines at a time
  const char* const plane = a.g.kv + (size_t)a.layer * a.g.plane_bytes + (PAGED ? 0 : (size_t)plan.seg_base[seg] * ROW);
  typedef const __attribute__((address_space(4))) int* const_int_p;
  const const_int_p pt = PAGED ? (const_int_p)(uintptr_t)(a.g.page_table + (size_t)req * a.g.pt_stride) : nullptr;
  const int pg_sh = PAGED ? a.g.pg_shift : 0, pg_mask = (1 << pg_sh) - 1;
  const int g8 = wave & 3;                         // rows g8 * 8 .. + 7 of a tile
  constexpr int U = DR / 8;                        // units of a rotated part: 8 rows are 64 of them, or (d_rope 32) 32
  int lofs[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) lofs[i] = (i * 4 + kg) * ROW + (l15 ^ swap256(g8 * 8 + i * 4 + kg)) * 16;
  const int rrow = (lane / U) & 7;
  const int rofs = rrow * ROW + DC * 2 + ((lane % U) ^ (U == 8 ? swap128(g8 * 8 + rrow) : swap64(g8 * 8 + rrow))) * 16;
  auto rows_at = [&](const char* p, int n) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, n * ROW, 0x00020000); };
  auto rows_of = [&](int tile) {
    const int at = c0 + tile * LK + g8 * 8, n = uni(tile < tiles ? max(0, min(8, span - at)) : 0);      // (no rows: zeros, without an access)
    const int t0 = uni(n > 0 ? at : 0);
    const size_t slot = PAGED ? ((size_t)pt[t0 >> pg_sh] << pg_sh) + (t0 & pg_mask) : (size_t)t0;
    return rows_at(plane + slot * ROW, n);
  };
  constexpr int LOADS = SUB * 2 + 1;
  auto load = [&](__amdgpu_buffer_rsrc_t buf, char* t, int i) {
    if (i < SUB * 2) load_to_lds(buf, t + (i >> 1) * SUB_B + (g8 * 8 + (i & 1) * 4) * 256, lofs[i & 1], (i >> 1) * 256);
    else if (DR == 64 || lane < 32) load_to_lds(buf, t + SUB * SUB_B + g8 * 8 * DR * 2, rofs, 0);
  };
  auto load_all = [&](__amdgpu_buffer_rsrc_t buf, char* t) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(buf, t, i);
  };
  load_all(rows_of(wave < 4 ? 0 : 1), wave < 4 ? s_0 : s_1);
  if constexpr (STAGED) {
    const int q0 = qb * R + (wave >> 2) * 32 + g8 * 8;
    load_all(rows_at(reinterpret_cast<const char*>(a.q) + ((size_t)row0 * H + q0) * ROW, uni(max(0, min(8, nq - q0)))), wave < 4 ? s_2 : s_3);
  }
  // scores: TQ x 16 rows x 16 slots of every tile a wave
  const int rg = wave & 1, kb = (wave >> 1) & 1, row = rg * 16 * TQ + l15;
  u32x4_t qf[TQ][NS];
  if (!STAGED && wave < 4) {
#pragma unroll
    for (int t = 0; t < TQ; ++t) {
      const bf16_t* q = a.q + ((size_t)row0 * H + min(qb * R + row + t * 16, nq - 1)) * (DC + DR) + kg * 8;
#pragma unroll
      for (int s = 0; s < NS; ++s) qf[t][s] = *reinterpret_cast<const u32x4_t*>(q + s * 32);
    }
  }
  if (c1 > P) {
    const float inv_H = 1.f / (float)H;
    for (int i = threadIdx.x; i < R * 12; i += 64 * LW) {
      const int r = i / 12, w = i - r * 12, qi = min(qb * R + r, nq - 1), node = (int)(((float)qi + 0.5f) * inv_H);
      s_anc[r][w] = w >= 1 && w <= 8 ? reinterpret_cast<const uint32_t*>(a.tables[req].anc[plan.seg_first[seg] + node])[w - 1] : 0u;
    }
  }
  if (threadIdx.x == 0) s_redo = 0;
  auto lds_done = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  SP_WAIT_VMEM(0);
  lds_done();
  bare_barrier();

  const float sc = a.scale * 1.4426950408889634f;
  constexpr float NONE = 3.4028234663852886e38f;
  // The weight of a score s is exp2(s * sc + shift): the shift is minus a past maximum of the row's s * sc.  It is changed at the first
  // tile, and at one where the row has weights past 2^FAR; the tile is then taken again.
  constexpr float FAR = 16.f;
  auto shifted = [&](int row, float shift) {
    const float top = fmaxf(s_max[row][0], s_max[row][1]) * sc;
    return top + shift > FAR ? -top : shift;
  };

  if (wave < 4) {
    // ---- scores
    // places of the lane's units: row l15 of sixteen, columns kg * 8 .. + 7 of 32
    const int ka = l15 * 256 + (kg ^ swap256(l15)) * 16, kr = SUB * SUB_B + l15 * DR * 2 + (kg ^ (DR == 64 ? swap128(l15) : swap64(l15))) * 16;
    auto unit = [&](const char* t, int sixteen, int s) {         // of rows sixteen * 16 .. of a tile
      return s < SUB * 4 ? *reinterpret_cast<const u32x4_t*>(t + sixteen * 4096 + (ka ^ ((s & 3) * 64)) + (s >> 2) * SUB_B)
                         : *reinterpret_cast<const u32x4_t*>(t + sixteen * 16 * DR * 2 + (kr ^ ((s - SUB * 4) * 64)));
    };
    if constexpr (STAGED) {
#pragma unroll
      for (int t = 0; t < TQ; ++t)
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[t][s] = unit(rg ? s_3 : s_2, t, s);
      lds_done();
      bare_barrier();                              // (the query rows' place is free)
    }
    const int pp = row * 64 + ((kb * 2 + (kg >> 1)) ^ swap64(row)) * 16 + (kg & 1) * 8;      // (row + 16: 1024 behind)
    float shift[TQ], sum[TQ], add[TQ];
    f32x4_t sa[TQ], sb[TQ];                        // scores of even and odd tiles
    bool bad_a = false, bad_b = false;             // what some rows do not see may not be finite
#pragma unroll
    for (int t = 0; t < TQ; ++t) { shift[t] = NONE; sum[t] = add[t] = 0.f; }
    float low;                                     // the lane's smallest exponent of the tile whose weights were formed last
    auto weights = [&](const f32x4_t (&sv)[TQ], int i) {         // of tile i; returns the largest exponent
      float top = -INFINITY;
      low = INFINITY;
#pragma unroll
      for (int t = 0; t < TQ; ++t) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(sv[t][j], sc, shift[t]);
        top = fmaxf(fmaxf(fmaxf(top, x[0]), fmaxf(x[1], x[2])), x[3]);
        low = fminf(fminf(fminf(low, x[0]), fminf(x[1], x[2])), x[3]);
        uint2 w;
        w.x = pack_bf16x2(__builtin_amdgcn_exp2f(x[0]), __builtin_amdgcn_exp2f(x[1]));
        w.y = pack_bf16x2(__builtin_amdgcn_exp2f(x[2]), __builtin_amdgcn_exp2f(x[3]));
        *reinterpret_cast<uint2*>(s_p[i & 1] + pp + t * 1024) = w;
        add[t] = dot2(w.x, dot2(w.y, 0.f));
      }
      return top;
    };
    // everyone sees the wave's sixteen slots of tile i
    auto all_seen = [&](int i) { const int k1 = c0 + i * LK + kb * 16 + 16; return k1 <= P && k1 <= c1; };
    // tile i on `cur`, and behind its scores the tile before, on `prev`, taken again where that is asked for
    auto step = [&](char* prev, const f32x4_t (&before)[TQ], bool bad_before, const char* cur, f32x4_t (&sv)[TQ], bool& bad, int i) {
      const int redo = s_redo;
      if (i < tiles) {
        constexpr int AHEAD = 6;
        u32x4_t kf[AHEAD];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) kf[s] = unit(cur, kb, s);
#pragma unroll
        for (int t = 0; t < TQ; ++t) sv[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
          for (int t = 0; t < TQ; ++t) sv[t] = mfma16(kf[s % AHEAD], qf[t][s], sv[t]);
          if (s + AHEAD < NS) kf[s % AHEAD] = unit(cur, kb, s + AHEAD);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD + 1, 0);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, TQ, 0);
          if (s + AHEAD < NS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      if (i > 0 && uni(redo) == i - 1) {
#pragma unroll
        for (int t = 0; t < TQ; ++t) {
          const float mx = quad_rows_max(fmaxf(fmaxf(before[t][0], before[t][1]), fmaxf(before[t][2], before[t][3])));
          if (kg == 0) s_max[row + t * 16][kb] = mx;
        }
        lds_done();
        bare_barrier();                            // maxima are posted
#pragma unroll
        for (int t = 0; t < TQ; ++t) {
          const float now = shifted(row + t * 16, shift[t]);
          sum[t] *= __builtin_amdgcn_exp2f(now - shift[t]);
          shift[t] = now;
        }
        weights(before, i - 1);
        if (all_seen(i - 1) ? __builtin_amdgcn_ballot_w64(low == -INFINITY) != 0 : bad_before) {
          // Values that are not finite count as nothing: for those who do not see them, and where the score is minus infinity.  Those who see
          // them have no other score but that, plus infinity or NaN, of which the last two make the weight NaN, and with it the row.
          for (int u = lane; u < SUB * 256; u += 64) {
            u32x4_t* p = reinterpret_cast<u32x4_t*>(prev + (u >> 8) * SUB_B + kb * 4096) + (u & 255);
            u32x4_t v = *p;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((v[j] & 0x7f80u) == 0x7f80u) v[j] &= 0xffff0000u;
              if ((v[j] & 0x7f800000u) == 0x7f800000u) v[j] &= 0x0000ffffu;
            }
            *p = v;
          }
        }
        lds_done();
        bare_barrier();                            // weights are posted
      }
#pragma unroll
      for (int t = 0; t < TQ; ++t) sum[t] += add[t];
      if (i >= tiles) return;
      const int k0 = c0 + i * LK + kb * 16;
      const bool all = all_seen(i);
      bad = false;
      if (!all) {
        // (what is not finite in a row of the cache shows in all of its scores)
        float odd = 0.f;
#pragma unroll
        for (int t = 0; t < TQ; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) odd += sv[t][j] * 0.f;
        bad = __builtin_amdgcn_ballot_w64(odd != odd) != 0;
        const int n0 = k0 - P;
#pragma unroll
        for (int t = 0; t < TQ; ++t) {
          uint32_t seen = low_bits(-n0);
          if (n0 > -32) {
            const uint32_t* w = &s_anc[row + t * 16][(n0 >> 5) + 1];
            seen |= __builtin_amdgcn_alignbit(w[1], w[0], n0 & 31);
          }
          seen = (seen & low_bits(c1 - k0)) >> (kg * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) sv[t][j] = (seen >> j) & 1u ? sv[t][j] : -INFINITY;
        }
      }
      if (i > 0) {                                 // (the first tile is taken again anyway)
        // Where everyone sees the slots, only an exponent of minus infinity leaves a row that their values could spoil: it is brought to plus
        // infinity, or NaN where the largest is no other, and added (in a bool beside the comparison: 26.0 -> 27.3 us a call, 64 nodes x 32
        // heads behind 2048; this way 26.0).
        const float top = weights(sv, i), far = __builtin_fmaf(all ? low : 0.f, -1e-37f, top);
        if ((bad || __builtin_amdgcn_ballot_w64(!(far <= FAR))) && lane == 0) s_redo = i;
      }
      lds_done();
      bare_barrier();                              // the tile's weights are there, the next tile is, nobody reads the one before
    };
    for (int i = 0; i <= tiles; i += 4) {
      step(s_3, sb, bad_b, s_0, sa, bad_a, i);
      if (i + 1 <= tiles) step(s_0, sa, bad_a, s_1, sb, bad_b, i + 1);
      if (i + 2 <= tiles) step(s_1, sb, bad_b, s_2, sa, bad_a, i + 2);
      if (i + 3 <= tiles) step(s_2, sa, bad_a, s_3, sb, bad_b, i + 3);
    }
#pragma unroll
    for (int t = 0; t < TQ; ++t) {
      const float l = quad_rows_sum(sum[t]);
      if (kg == 0) s_max[row + t * 16][kb] = l;
    }
    lds_done();
    bare_barrier();
    return;
  }

  // ---- results: CG x 64 columns of all rows, one tile behind the scores; and the tiles to come
  const int l31 = lane & 31, h = lane >> 5, b = (lane >> 4) & 1, r = l15 >> 2, c = l15 & 3;
  const int c64 = g8 * CG;                         // the wave's first 64 columns
  f32x16_t o[CG][2][RT];
#pragma unroll
  for (int g = 0; g < CG; ++g)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[g][e][t][j] = 0.f;
  float shift[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) shift[t] = NONE;
  // places of the lane's transposing reads (unit of 64 columns g: 8 units on, and 128 columns a sub-tile) and of its weights
  const int va = (h * 8 + r) * 256 + ((b * 4 + c) ^ swap256(h * 8 + r)) * 16 + b * 8;
  const int pa = l31 * 64 + (h ^ swap64(l31)) * 16;
  if constexpr (STAGED) bare_barrier();            // (the query rows' place is free)
  auto next_tile = [&] {
    SP_WAIT_VMEM(LOADS);
    lds_done();
    bare_barrier();                                // the tile's weights are there, the next tile is, nobody reads the one before
  };
  // the loads of tile i + 2 into `next`, the weights of tile i - 1 on `cur`
  auto step = [&](const char* cur, char* next, int i) {
    const int redo = s_redo;
    const auto buf = rows_of(i + 2);
    if (uni(redo) == i - 1) {
      bare_barrier();                            // maxima are posted
      bool any = false;
      float by[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float now = shifted(t * 32 + l31, shift[t]);
        any = any || now != shift[t];
        by[t] = __builtin_amdgcn_exp2f(now - shift[t]);
        shift[t] = now;
      }
      if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
        for (int g = 0; g < CG; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int t = 0; t < RT; ++t) o[g][e][t] *= by[t];
      }
      lds_done();
      bare_barrier();                            // weights are posted
    }
    // The loads go out among the products: one after the other they hold the wave up, 64 bytes a clock is all that a CU takes.
    const char* pw = s_p[(i - 1) & 1];
    constexpr int N = LK / 16 * CG * 2;
    u32x4_t p[LK / 16][RT];
#pragma unroll
    for (int k = 0; k < LK / 16; ++k)
#pragma unroll
      for (int t = 0; t < RT; ++t) p[k][t] = *reinterpret_cast<const u32x4_t*>(pw + (pa ^ (k * 32)) + t * 2048);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int k = n / (CG * 2), g = n / 2 % CG, e = n & 1;
      const int at = (va ^ (e * 8) ^ (((c64 + g) & 1) * 128)) + ((c64 + g) >> 1) * SUB_B + k * 4096;
      const uint2 lo = read_transposed(cur + at), hi = read_transposed(cur + (at ^ 16) + 1024);
      const u32x4_t v = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
      for (int t = 0; t < RT; ++t) o[g][e][t] = mfma32(v, p[k][t], o[g][e][t]);
      load(buf, next, n);
    }
    static_assert(LOADS == N + 1, "a load for every fragment, and one");
    load(buf, next, N);
    __builtin_amdgcn_sched_group_barrier(0x100, LK / 16 * RT + 4, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      __builtin_amdgcn_sched_group_barrier(0x008, RT, 0);
      if (n + 2 < N) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
    }
    next_tile();
  };
  load_all(rows_of(2), s_2);
  next_tile();
  for (int i = 1;;) {
    step(s_0, s_3, i);
    if (++i > tiles) break;
    step(s_1, s_0, i);
    if (++i > tiles) break;
    step(s_2, s_1, i);
    if (++i > tiles) break;
    step(s_3, s_2, i);
    if (++i > tiles) break;
  }
  SP_WAIT_VMEM(0);                                 // (zeros, on their way to a place that the workgroup gives away)

#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = t * 32 + l31, qi = qb * R + row;
    if (qi >= nq) continue;
    const float l = s_max[row][0] + s_max[row][1], inv = 1.f / l;
    const size_t at = (size_t)plan.seg_unit0[seg] + (size_t)ch * nq + qi;
    // o[g][e][t][4 j ..]: columns (c64 + g) * 64 + (j / 2) * 32 + ((j & 1) * 2 + h) * 8 + (e ^ j / 2) * 4 ..
#pragma unroll
    for (int g = 0; g < CG; ++g)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int f = j >> 1, col = (c64 + g) * 64 + f * 32 + ((j & 1) * 2 + h) * 8;
        f32x4_t x = {o[g][f][t][j * 4], o[g][f][t][j * 4 + 1], o[g][f][t][j * 4 + 2], o[g][f][t][j * 4 + 3]};
        f32x4_t y = {o[g][1 - f][t][j * 4], o[g][1 - f][t][j * 4 + 1], o[g][1 - f][t][j * 4 + 2], o[g][1 - f][t][j * 4 + 3]};
        if (chunks == 1) {
          x *= inv; y *= inv;
          *reinterpret_cast<u32x4_t*>(a.out + ((size_t)row0 * H + qi) * DC + col) =
              (u32x4_t){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        } else {
          float* po = a.part + at * DC + col;
          *reinterpret_cast<f32x4_t*>(po) = x;
          *reinterpret_cast<f32x4_t*>(po + 4) = y;
        }
      }
    if (chunks > 1 && c64 == 0 && h == 0) {
      float* ml = a.part + (size_t)plan.units_total * DC + at * 2;
      ml[0] = -shift[t]; ml[1] = l;
    }
  }
}

// A query row of the call, row * H + head: the request it belongs to, and its partial rows.
struct LatentRow { int chunks; size_t u0, stride; };
__device__ __forceinline__ LatentRow latent_row(const AttnPlan& plan, int at, int H, int lane) {
  const int row = at / H;
  int seg = 0;
  if (plan.n_seg > 1) {
    const int first = plan.seg_row0[lane];
    seg = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(lane < plan.n_seg && row >= first && row < first + plan.seg_rows[lane])) - 1;
  }
  return {plan.seg_chunks[seg], (size_t)plan.seg_unit0[seg] + at - (size_t)plan.seg_row0[seg] * H, (size_t)plan.seg_rows[seg] * H};
}

// Chunks j of a row, results o_j, sums l_j, shifts m_j: out = sum_j w_j o_j / sum_j w_j l_j with w_j = exp2(m_j - max m).  Bound by the
// partial rows' way in.  Few chunks: a wave joins those of a query row, DC / 64 columns a lane, four chunks on their way at a time (8192
// rows of two chunks 8.7 us, 33 MB; the 16 to 128 rows of 32 requests in up to four 5.4; with the kernel for many 19.6 and 9.3).
#define LATENT_FEW 16
template <int DC>
__global__ void __launch_bounds__(256) k_latent_merge_few(LatentAttnArgs a, AttnPlan plan, int at0, int n) {
  constexpr int V = DC / 256;                      // four columns at lane * 4 + 256 v
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at = at0 + blockIdx.x * 4 + wave;
  if (at >= n) return;
  const LatentRow r = latent_row(plan, at, a.d.n_heads, lane);
  if (r.chunks == 1) return;
  const float* ml = a.part + (size_t)plan.units_total * DC;
  float m = -INFINITY, s = 0.f;
  if (lane < r.chunks) {
    const float2 x = *reinterpret_cast<const float2*>(ml + (r.u0 + lane * r.stride) * 2);
    m = x.x; s = x.y;
  }
  const float* po = a.part + r.u0 * DC + lane * 4;
  f32x4_t acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  float w = 0.f;
  for (int j = 0; j < r.chunks; j += 4) {
    f32x4_t x[4][V];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) x[i][v] = *reinterpret_cast<const f32x4_t*>(po + (size_t)min(j + i, r.chunks - 1) * r.stride * DC + v * 256);
    if (j == 0) w = __builtin_amdgcn_exp2f(m - wave_max(m));     // (lanes without a chunk: zero)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float wi = __shfl(w, j + i, 64);       // (none: zero)
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] += wi * x[i][v];
    }
  }
  const float inv = 1.f / wave_sum(w * s);
#pragma unroll
  for (int v = 0; v < V; ++v)
    *reinterpret_cast<uint2*>(a.out + (size_t)at * DC + lane * 4 + v * 256) =
        uint2{pack_bf16x2(acc[v][0] * inv, acc[v][1] * inv), pack_bf16x2(acc[v][2] * inv, acc[v][3] * inv)};
}

// Many: a workgroup joins those of a query row, a thread four columns, groups of threads every second chunk (DC 256: fourth), eight on
// their way at a time (80 rows of 64 chunks 5.2 us; with the kernel for few 14.4).
template <int DC>
__global__ void __launch_bounds__(256) k_latent_merge(LatentAttnArgs a, AttnPlan plan, int at0) {
  constexpr int T = DC / 4, G = 256 / T;           // threads of a row, groups of chunks
  __shared__ float s_w[256], s_red[8];
  __shared__ __attribute__((aligned(16))) float s_acc[(G - 1) * DC];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at = at0 + blockIdx.x;
  const LatentRow r = latent_row(plan, at, a.d.n_heads, lane);
  if (r.chunks == 1) return;
  const int chunks = r.chunks;
  const size_t stride = r.stride, u0 = r.u0;
  const float* ml = a.part + (size_t)plan.units_total * DC;
  const int col = (threadIdx.x % T) * 4, group = threadIdx.x / T;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f, mx = -INFINITY;
  for (int b = 0; b < chunks; b += 256) {
    const int nb = min(256, chunks - b);
    float m = -INFINITY, s = 0.f;
    if ((int)threadIdx.x < nb) {
      const float2 x = *reinterpret_cast<const float2*>(ml + (u0 + (b + threadIdx.x) * stride) * 2);
      m = x.x; s = x.y;
    }
    const float wm = wave_max(m);
    if (lane == 0) s_red[wave] = wm;
    __syncthreads();
    const float top = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), mx);
    const float f = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - top), w = (int)threadIdx.x < nb ? __builtin_amdgcn_exp2f(m - top) : 0.f;
    s_w[threadIdx.x] = w;
    const float ws = wave_sum(w * s);
    if (lane == 0) s_red[4 + wave] = ws;
    __syncthreads();
    l = l * f + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
    acc *= f;
    mx = top;
    const float* po = a.part + (u0 + (size_t)b * stride) * DC + col;
    int j = group;
    for (; j + 7 * G < nb; j += 8 * G) {
      f32x4_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(po + (size_t)(j + i * G) * stride * DC);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc += s_w[j + i * G] * x[i];
    }
    for (; j < nb; j += G) acc += s_w[j] * *reinterpret_cast<const f32x4_t*>(po + (size_t)j * stride * DC);
    __syncthreads();
  }
  if (group > 0) *reinterpret_cast<f32x4_t*>(s_acc + (group - 1) * DC + col) = acc;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 1; g < G; ++g) acc += *reinterpret_cast<const f32x4_t*>(s_acc + (g - 1) * DC + col);
  const float inv = 1.f / l;
  *reinterpret_cast<uint2*>(a.out + (size_t)at * DC + col) = uint2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
}

bool sp_latent_attn_covers(const LatentDims& d) { return (d.d_latent == 512 || d.d_latent == 256) && (d.d_rope == 64 || d.d_rope == 32); }

template <int DC, int DR, int R>
static hipError_t go(const LatentAttnArgs& a, const AttnPlan& plan, int M, hipStream_t st) {
  const dim3 grid(plan.total_items), block(64 * LW);
  if (a.g.page_table) hipLaunchKernelGGL((k_latent_attn<DC, DR, R, true>), grid, block, 0, st, a, plan);
  else hipLaunchKernelGGL((k_latent_attn<DC, DR, R, false>), grid, block, 0, st, a, plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !plan.any_split) return e;
  const int n = M * a.d.n_heads;
  int most = 0;
  for (int i = 0; i < plan.n_seg; ++i) most = plan.seg_chunks[i] > most ? plan.seg_chunks[i] : most;
  // (in several launches where there are more query rows than a grid takes)
  for (int at0 = 0; at0 < n; at0 += 1 << 23) {
    const int rows = n - at0 < 1 << 23 ? n - at0 : 1 << 23;
    if (most <= LATENT_FEW) hipLaunchKernelGGL((k_latent_merge_few<DC>), dim3((rows + 3) / 4), dim3(256), 0, st, a, plan, at0, n);
    else hipLaunchKernelGGL((k_latent_merge<DC>), dim3(rows), dim3(256), 0, st, a, plan, at0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int DC, int DR>
static hipError_t go(const LatentAttnArgs& a, const AttnPlan& plan, int M, hipStream_t st) {
  return plan.qt == 2 ? go<DC, DR, 32>(a, plan, M, st) : plan.qt == 4 ? go<DC, DR, 64>(a, plan, M, st) : hipErrorInvalidValue;
}
hipError_t sp_launch_latent_attn(const LatentAttnArgs& a, const AttnPlan& plan, int M, hipStream_t st) {
  if (a.g.row_bytes != (a.d.d_latent + a.d.d_rope) * 2) return hipErrorInvalidValue;
  if (a.d.d_latent == 512 && a.d.d_rope == 64) return go<512, 64>(a, plan, M, st);
  if (a.d.d_latent == 512 && a.d.d_rope == 32) return go<512, 32>(a, plan, M, st);
  if (a.d.d_latent == 256 && a.d.d_rope == 64) return go<256, 64>(a, plan, M, st);
  if (a.d.d_latent == 256 && a.d.d_rope == 32) return go<256, 32>(a, plan, M, st);
  return hipErrorInvalidValue;
}
