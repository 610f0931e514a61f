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
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

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
  __shared__ __attribute__((aligned(16))) char s_0[TILE], s_1[TILE], s_2[TILE], s_3[TILE];
  __shared__ __attribute__((aligned(16))) char s_p[2][R * LK * 2];
  __shared__ __attribute__((aligned(16))) float s_max[R][2];
  __shared__ uint32_t s_anc[R][12];                // ancestor masks of the query rows, a word of zeros in front, three behind
  __shared__ int s_redo;

  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, kg = lane >> 4;
  const int item = blockIdx.x;
  int seg = 0;
  if (plan.n_seg > 1) seg = uni(__popcll(__builtin_amdgcn_ballot_w64(lane < plan.n_seg && item >= plan.seg_item0[lane])) - 1);
  const int chunks = plan.seg_chunks[seg], seg_rows = plan.seg_rows[seg], row0 = plan.seg_row0[seg], req = plan.seg_req[seg];
  const int P = plan.seg_P[seg], span = P + plan.seg_T[seg], clen = plan.seg_clen[seg];
  const int local = item - plan.seg_item0[seg], qb = uni(local / chunks), ch = local - qb * chunks;
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
    const int at = c0 + tile * LK + g8 * 8, n = uni(max(0, min(8, span - at)));
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
  {
    const int q0 = qb * R + (R == 64 && wave >= 4 ? 32 : 0) + g8 * 8;
    const auto buf = rows_at(reinterpret_cast<const char*>(a.q) + ((size_t)row0 * H + q0) * ROW, uni(max(0, min(8, nq - q0))));
    if (wave < 4) {
      load_all(buf, s_2);
      load_all(rows_of(0), s_0);
    } else {
      if (R == 64) load_all(buf, s_3);
      load_all(rows_of(1), s_1);
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
    // ---- scores: 32 rows x 16 slots of every tile
    const bool on = R == 64 || wave < 2;
    const int rg = R == 64 ? wave & 1 : 0, kb = R == 64 ? wave >> 1 : wave & 1;
    // places of the lane's units: row l15 of sixteen, columns kg * 8 .. + 7 of 32
    const int ka = l15 * 256 + (kg ^ swap256(l15)) * 16, kr = SUB * SUB_B + l15 * DR * 2 + (kg ^ (DR == 64 ? swap128(l15) : swap64(l15))) * 16;
    auto unit = [&](const char* t, int s) {
      return s < SUB * 4 ? *reinterpret_cast<const u32x4_t*>(t + (ka ^ ((s & 3) * 64)) + (s >> 2) * SUB_B)
                         : *reinterpret_cast<const u32x4_t*>(t + (kr ^ ((s - SUB * 4) * 64)));
    };
    u32x4_t qf[2][NS];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int at = s < SUB * 4 ? t * 4096 : t * 16 * DR * 2;
        qf[t][s] = unit((rg ? s_3 : s_2) + at, s);
      }
    lds_done();
    bare_barrier();                                // (the query rows' place is free)
    float shift[2] = {NONE, NONE}, sum[2] = {0.f, 0.f};
    const int row = rg * 32 + l15;
    const int pp = row * 64 + ((kb * 2 + (kg >> 1)) ^ swap64(row)) * 16 + (kg & 1) * 8;      // (row + 16: 1024 behind)
    auto step = [&](const char* cur, int i) {
      if (!on) { lds_done(); bare_barrier(); if (uni(s_redo) == i) { bare_barrier(); bare_barrier(); } return; }
      const int k0 = c0 + i * LK + kb * 16;
      f32x4_t sv[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      {
        constexpr int AHEAD = 6;
        u32x4_t kf[AHEAD];
        auto key = [&](int s) { return unit(cur + (s < SUB * 4 ? kb * 4096 : kb * 16 * DR * 2), s); };
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) kf[s] = key(s);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
          for (int t = 0; t < 2; ++t) sv[t] = mfma16(kf[s % AHEAD], qf[t][s], sv[t]);
          if (s + AHEAD < NS) kf[s % AHEAD] = key(s + AHEAD);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
          if (s + AHEAD < NS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      bool bad = false;
      if (k0 + 16 > P || k0 + 16 > c1) {
        // (what is not finite in a row of the cache shows in all of its scores)
        float odd = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) odd += sv[t][j] * 0.f;
        bad = __builtin_amdgcn_ballot_w64(odd != odd) != 0;
        const int n0 = k0 - P;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
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
      float add[2], top = -INFINITY;
      auto weights = [&] {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(sv[t][j], sc, shift[t]);
          top = fmaxf(fmaxf(fmaxf(top, x[0]), fmaxf(x[1], x[2])), x[3]);
          uint2 w;
          w.x = pack_bf16x2(__builtin_amdgcn_exp2f(x[0]), __builtin_amdgcn_exp2f(x[1]));
          w.y = pack_bf16x2(__builtin_amdgcn_exp2f(x[2]), __builtin_amdgcn_exp2f(x[3]));
          add[t] = (bf16_lo(w.x) + bf16_hi(w.x)) + (bf16_lo(w.y) + bf16_hi(w.y));
          *reinterpret_cast<uint2*>(s_p[i & 1] + pp + t * 1024) = w;
        }
      };
      weights();
      if ((bad || __builtin_amdgcn_ballot_w64(top > FAR)) && lane == 0) s_redo = i;
      lds_done();
      bare_barrier();                              // the tile's weights are there, the next tile is, nobody reads the one before
      if (uni(s_redo) == i) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float mx = quad_rows_max(fmaxf(fmaxf(sv[t][0], sv[t][1]), fmaxf(sv[t][2], sv[t][3])));
          if (kg == 0) s_max[row + t * 16][kb] = mx;
        }
        lds_done();
        bare_barrier();                            // maxima are posted
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float now = shifted(row + t * 16, shift[t]);
          sum[t] *= __builtin_amdgcn_exp2f(now - shift[t]);
          shift[t] = now;
        }
        weights();
        if (bad) {
          // values that are not finite count as nothing for those who do not see them (those who do have scores that are none)
          for (int u = lane; u < SUB * 256; u += 64) {
            u32x4_t* p = reinterpret_cast<u32x4_t*>(const_cast<char*>(cur) + (u >> 8) * SUB_B + kb * 4096) + (u & 255);
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
        bare_barrier();
      }
      sum[0] += add[0];
      sum[1] += add[1];
    };
    for (int i = 0; i < tiles; i += 4) {
      step(s_0, i);
      if (i + 1 < tiles) step(s_1, i + 1);
      if (i + 2 < tiles) step(s_2, i + 2);
      if (i + 3 < tiles) step(s_3, i + 3);
    }
    if (on) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float l = quad_rows_sum(sum[t]);
        if (kg == 0) s_max[row + t * 16][kb] = l;
      }
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
  bare_barrier();                                  // (the query rows' place is free)
  // the weights of tile i - 1 on `cur`, the loads of tile i + 2 into `next`; then tile i's weights
  auto step = [&](const char* cur, char* next, int i) {
    const bool more = i + 2 < tiles;
    const auto buf = rows_of(more ? i + 2 : 0);
    if (i > 0) {
      const char* pw = s_p[(i - 1) & 1];
#pragma unroll
      for (int k = 0; k < LK / 16; ++k) {
        u32x4_t p[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) p[t] = *reinterpret_cast<const u32x4_t*>(pw + (pa ^ (k * 32)) + t * 2048);
#pragma unroll
        for (int g = 0; g < CG; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int at = (va ^ (e * 8) ^ (((c64 + g) & 1) * 128)) + ((c64 + g) >> 1) * SUB_B + k * 4096;
            const uint2 lo = read_transposed(cur + at), hi = read_transposed(cur + (at ^ 16) + 1024);
            const u32x4_t v = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
            for (int t = 0; t < RT; ++t) o[g][e][t] = mfma32(v, p[t], o[g][e][t]);
          }
      }
    }
    if (more) {
      load_all(buf, next);
      SP_WAIT_VMEM(LOADS);
    } else {
      SP_WAIT_VMEM(0);
    }
    lds_done();
    bare_barrier();                                // the tile's weights are there, the next tile is, nobody reads the one before
    if (i < tiles && uni(s_redo) == i) {
      bare_barrier();                              // maxima are posted
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
      bare_barrier();
    }
  };
  for (int i = 0; i <= tiles; i += 4) {
    step(s_3, s_2, i);
    if (i + 1 <= tiles) step(s_0, s_3, i + 1);
    if (i + 2 <= tiles) step(s_1, s_0, i + 2);
    if (i + 3 <= tiles) step(s_2, s_1, i + 3);
  }

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

// A wave joins the chunks of a query row, DC / 64 columns a lane: first every lane one chunk's weight, then the rows in their order.
template <int DC>
__global__ void __launch_bounds__(256) k_latent_merge(LatentAttnArgs a, AttnPlan plan, int n) {
  constexpr int V = DC / 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, H = a.d.n_heads;
  const int at = blockIdx.x * 4 + wave;            // row * H + head of the call
  if (at >= n) return;
  const int row = at / H;
  int seg = 0;
  if (plan.n_seg > 1) {
    const int first = plan.seg_row0[lane];
    seg = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(lane < plan.n_seg && row >= first && row < first + plan.seg_rows[lane])) - 1;
  }
  const int chunks = plan.seg_chunks[seg];
  if (chunks == 1) return;
  const size_t stride = (size_t)plan.seg_rows[seg] * H, u0 = (size_t)plan.seg_unit0[seg] + at - (size_t)plan.seg_row0[seg] * H;
  const float* ml = a.part + (size_t)plan.units_total * DC;
  float acc[V], l = 0.f, mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  for (int b = 0; b < chunks; b += 64) {
    float m = -INFINITY, s = 0.f;
    if (b + lane < chunks) {
      const float2 x = *reinterpret_cast<const float2*>(ml + (u0 + (b + lane) * stride) * 2);
      m = x.x; s = x.y;
    }
    const float top = fmaxf(mx, wave_max(m)), f = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - top);
    l *= f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] *= f;
    mx = top;
    const float w = b + lane < chunks ? __builtin_amdgcn_exp2f(m - top) : 0.f;
    l += wave_sum(w * s);
    const int nb = min(64, chunks - b);
    for (int j = 0; j < nb; ++j) {
      const float wj = __shfl(w, j, 64);
      const float* po = a.part + (u0 + (size_t)(b + j) * stride) * DC + lane * V;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(po + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i + e] += wj * x[e];
      }
    }
  }
  const float inv = 1.f / l;
  bf16_t* out = a.out + (size_t)at * DC + lane * V;
#pragma unroll
  for (int i = 0; i < V; i += 4)
    *reinterpret_cast<uint2*>(out + i) = uint2{pack_bf16x2(acc[i] * inv, acc[i + 1] * inv), pack_bf16x2(acc[i + 2] * inv, acc[i + 3] * inv)};
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
  hipLaunchKernelGGL((k_latent_merge<DC>), dim3((n + 3) / 4), dim3(256), 0, st, a, plan, n);
  return hipGetLastError();
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
