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

#define LW 8                       // waves per workgroup
#define LK 64                      // slots per tile

// Places of 16-byte units in LDS: rows of 256 bytes, and rows of 128 or 64.
__device__ __forceinline__ int swap256(int row) { return (row & 3) * 4 + ((row >> 2) & 3); }
__device__ __forceinline__ int swap128(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swap64(int row) { return (row >> 2) & 3; }

// A value that the compiler takes for another one each time: what is computed from it is computed again, not kept in registers.
__device__ __forceinline__ int again(int v) { asm volatile("" : "+v"(v)); return v; }

// R query rows (32 or 64) per workgroup.
template <int DC, int DR, int R, bool PAGED>
__global__ void __launch_bounds__(64 * LW, 2) k_latent_attn(LatentAttnArgs a, AttnPlan plan) {
  constexpr int SUB = DC / 128, ROW = (DC + DR) * 2, KR = DR / 32, NS = DC / 32 + KR;
  constexpr int SUB_B = LK * 256, TILE = SUB * SUB_B + LK * DR * 2;
  // results: 64 columns x RT blocks of 32 rows a wave
  constexpr int PW = DC / 64, RT = R / 32 * PW > LW ? 2 : 1;
  constexpr bool HALVED = RT == 1 && R == 64;                    // two waves share 64 columns
  __shared__ __attribute__((aligned(16))) char s_a[TILE], s_b[TILE];
  __shared__ __attribute__((aligned(16))) char s_p[R * LK * 2];
  __shared__ __attribute__((aligned(16))) float s_max[2][R][4];
  __shared__ uint32_t s_anc[R][12];                // ancestor masks of the query rows, a word of zeros in front, three behind
  __shared__ int s_redo;

  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int item = blockIdx.x;
  int seg = 0;
  if (plan.n_seg > 1) seg = uni(__popcll(__builtin_amdgcn_ballot_w64(lane < plan.n_seg && item >= plan.seg_item0[lane])) - 1);
  const int chunks = plan.seg_chunks[seg], seg_rows = plan.seg_rows[seg], row0 = plan.seg_row0[seg], req = plan.seg_req[seg];
  const int P = plan.seg_P[seg], span = P + plan.seg_T[seg], clen = plan.seg_clen[seg];
  const int local = item - plan.seg_item0[seg], qb = uni(local / chunks), ch = local - qb * chunks;
  const int H = a.d.n_heads, nq = seg_rows * H;    // query rows of the request, node * H + head
  const int c0 = ch * clen, c1 = min(c0 + clen, span);

  // a wave brings in rows 8 * wave .. + 7 of a tile
  const char* const plane = a.g.kv + (size_t)a.layer * a.g.plane_bytes + (PAGED ? 0 : (size_t)plan.seg_base[seg] * ROW);
  typedef const __attribute__((address_space(4))) int* const_int_p;
  const const_int_p pt = PAGED ? (const_int_p)(uintptr_t)(a.g.page_table + (size_t)req * a.g.pt_stride) : nullptr;
  const int pg_sh = PAGED ? a.g.pg_shift : 0, pg_mask = (1 << pg_sh) - 1;
  auto fetch = [&](char* t, int s0) {
    const int ln = again(lane), l15 = ln & 15, kg = ln >> 4;
    const int at = s0 + wave * 8, n = uni(max(0, min(8, span - at)));
    const int t0 = uni(n > 0 ? at : 0);
    const size_t slot = PAGED ? ((size_t)pt[t0 >> pg_sh] << pg_sh) + (t0 & pg_mask) : (size_t)t0;
    const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(plane) + slot * ROW, (short)0, n * ROW, 0x00020000);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int lofs = (i * 4 + kg) * ROW + (l15 ^ swap256(wave * 8 + i * 4 + kg)) * 16;
#pragma unroll
      for (int s = 0; s < SUB; ++s) load_to_lds(buf, t + s * SUB_B + (wave * 8 + i * 4) * 256, lofs, s * 256);
    }
    constexpr int U = DR / 8;                      // units of a rotated part: 8 rows are 64 of them, or (d_rope 32) 32
    const int r = (ln / U) & 7, row = wave * 8 + r;
    const int rofs = r * ROW + DC * 2 + ((ln % U) ^ (U == 8 ? swap128(row) : swap64(row))) * 16;
    if (DR == 64 || ln < 32) load_to_lds(buf, t + SUB * SUB_B + wave * 8 * DR * 2, rofs, 0);
  };
  fetch(s_a, c0);

  // ---- queries (scores: 32 rows x 16 slots a wave), ancestor masks
  const bool scores = R == 64 || wave < 4;
  const int rg = R == 64 ? wave & 1 : 0, kb = R == 64 ? wave >> 1 : wave & 3;
  u32x4_t qf[2][NS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bf16_t* qp = a.q + ((size_t)row0 * H + min(qb * R + rg * 32 + t * 16 + (lane & 15), nq - 1)) * (DC + DR) + (lane >> 4) * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[t][s] = *reinterpret_cast<const u32x4_t*>(qp + s * 32);
  }
  if (c1 > P) {
    const float inv_H = 1.f / (float)H;
    for (int i = threadIdx.x; i < R * 12; i += 64 * LW) {
      const int r = i / 12, w = i - r * 12, qi = min(qb * R + r, nq - 1), node = (int)(((float)qi + 0.5f) * inv_H);
      s_anc[r][w] = w >= 1 && w <= 8 ? reinterpret_cast<const uint32_t*>(a.tables[req].anc[plan.seg_first[seg] + node])[w - 1] : 0u;
    }
  }
  if (threadIdx.x == 0) s_redo = -1;

  const int pw = HALVED ? wave >> 1 : wave, pr = HALVED ? wave & 1 : 0;      // the wave's 64 columns and its first block of 32 rows
  const bool values = pw < PW;
  f32x16_t o[2][RT];
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[e][t][i] = 0.f;
  const float sc = a.scale * 1.4426950408889634f;
  constexpr float NONE = 3.4028234663852886e38f;
  float shift_s[2] = {NONE, NONE}, sum[2] = {0.f, 0.f}, shift_v[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) shift_v[t] = NONE;

  // par: the tile's number, odd or even
  auto tile = [&](const char* cur, char* other, int s0, int par) {
    SP_WAIT_VMEM(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    bare_barrier();                                // the tile is there whole, and nobody reads the other one any more
    if (s0 + LK < c1) fetch(other, s0 + LK);
    // The shift only has to keep the weights in range: it follows the maxima of the tile before, and where this tile's are out of
    // range (and at the first one) the tile is taken again with its own.
    auto lower = [&](int which, int row, float shift) {
      const f32x4_t m = *reinterpret_cast<const f32x4_t*>(s_max[which][row]);
      const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * sc;
      return top + shift > 8.f ? -top : shift;
    };
    for (bool own = s0 == c0;;) {
      const int ln = again(lane), l15 = ln & 15, kg = ln >> 4, k0 = s0 + kb * 16;
      f32x4_t sv[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      float add[2] = {0.f, 0.f};
      bool bad = false;
      if (scores) {
        const int ka = (kb * 16 + l15) * 256 + (kg ^ swap256(l15)) * 16;
        const int kr = SUB * SUB_B + (kb * 16 + l15) * DR * 2 + (kg ^ (DR == 64 ? swap128(kb * 16 + l15) : swap64(kb * 16 + l15))) * 16;
        constexpr int AHEAD = 4;
        u32x4_t kf[AHEAD];
        auto key = [&](int s) {
          return s < SUB * 4 ? *reinterpret_cast<const u32x4_t*>(cur + (ka ^ ((s & 3) * 64)) + (s >> 2) * SUB_B)
                             : *reinterpret_cast<const u32x4_t*>(cur + (kr ^ ((s - SUB * 4) * 64)));
        };
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
        if (k0 + 16 > P || k0 + 16 > c1) {
          // (what is not finite in a row of the cache shows in all of its scores)
          float odd = 0.f;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd += sv[t][i] * 0.f;
          bad = __builtin_amdgcn_ballot_w64(odd != odd) != 0;
          const int n0 = k0 - P;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t seen = low_bits(-n0);
            if (n0 > -32) {
              const uint32_t* w = &s_anc[rg * 32 + t * 16 + l15][(n0 >> 5) + 1];
              seen |= __builtin_amdgcn_alignbit(w[1], w[0], n0 & 31);
            }
            seen = (seen & low_bits(c1 - k0)) >> (kg * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) sv[t][i] = (seen >> i) & 1u ? sv[t][i] : -INFINITY;
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float mx = quad_rows_max(fmaxf(fmaxf(sv[t][0], sv[t][1]), fmaxf(sv[t][2], sv[t][3])));
          if (kg == 0) s_max[par][rg * 32 + t * 16 + l15][kb] = mx;
        }
      }
      if (own) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        bare_barrier();                            // maxima are posted, nobody reads the tile as keys any more
      }
      if (scores) {
        bool out = false;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int row = rg * 32 + t * 16 + l15;
          const float now = lower(own ? par : par ^ 1, row, shift_s[t]);
          sum[t] *= __builtin_amdgcn_exp2f(now - shift_s[t]);
          shift_s[t] = now;
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(sv[t][i], sc, now);
          out = out || fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) > 64.f;
          uint2 w;
          w.x = pack_bf16x2(__builtin_amdgcn_exp2f(x[0]), __builtin_amdgcn_exp2f(x[1]));
          w.y = pack_bf16x2(__builtin_amdgcn_exp2f(x[2]), __builtin_amdgcn_exp2f(x[3]));
          add[t] = (bf16_lo(w.x) + bf16_hi(w.x)) + (bf16_lo(w.y) + bf16_hi(w.y));
          *reinterpret_cast<uint2*>(s_p + row * 128 + ((kb * 2 + (kg >> 1)) ^ swap128(row)) * 16 + (kg & 1) * 8) = w;
        }
        if (!own && (bad || __builtin_amdgcn_ballot_w64(out)) && ln == 0) s_redo = s0;
        if (own && bad) {
          // values that are not finite count as nothing for those who do not see them (those who do have scores that are none)
          for (int i = ln; i < SUB * 256; i += 64) {
            u32x4_t* u = reinterpret_cast<u32x4_t*>(const_cast<char*>(cur) + (i >> 8) * SUB_B + kb * 4096) + (i & 255);
            u32x4_t v = *u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((v[j] & 0x7f80u) == 0x7f80u) v[j] &= 0xffff0000u;
              if ((v[j] & 0x7f800000u) == 0x7f800000u) v[j] &= 0x0000ffffu;
            }
            *u = v;
          }
        }
      }
      if (values) {
        bool any = false;
        float by[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float now = lower(own ? par : par ^ 1, (pr + t) * 32 + (ln & 31), shift_v[t]);
          any = any || now != shift_v[t];
          by[t] = __builtin_amdgcn_exp2f(now - shift_v[t]);
          shift_v[t] = now;
        }
        if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) o[e][t] *= by[t];
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      bare_barrier();                              // weights are posted
      if (own || uni(s_redo) != s0) {
        sum[0] += add[0];
        sum[1] += add[1];
        break;
      }
      own = true;
    }
    if (values) {
      const int ln = again(lane), l15 = ln & 15, h = ln >> 5, b = (ln >> 4) & 1, r = l15 >> 2, c = l15 & 3;
      const int va = (pw >> 1) * SUB_B + (h * 8 + r) * 256 + (((pw & 1) * 8 + b * 4 + c) ^ swap256(h * 8 + r)) * 16 + b * 8;
      const int pa = (pr * 32 + (ln & 31)) * 128 + (h ^ swap128(ln & 31)) * 16;
#pragma unroll
      for (int k = 0; k < LK / 16; ++k) {
        u32x4_t p[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) p[t] = *reinterpret_cast<const u32x4_t*>(s_p + (pa ^ (k * 32)) + t * 4096);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint2 lo = read_transposed(cur + (va ^ (e * 8)) + k * 4096), hi = read_transposed(cur + (va ^ (e * 8 + 16)) + 1024 + k * 4096);
          const u32x4_t v = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
          for (int t = 0; t < RT; ++t) o[e][t] = mfma32(v, p[t], o[e][t]);
        }
      }
    }
  };
  int s0 = c0;
  while (true) {
    tile(s_a, s_b, s0, 0);
    if ((s0 += LK) >= c1) break;
    tile(s_b, s_a, s0, 1);
    if ((s0 += LK) >= c1) break;
  }

  __syncthreads();                                 // (nobody reads maxima any more)
  if (scores) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float l = quad_rows_sum(sum[t]);
      if (lane < 16) s_max[0][rg * 32 + t * 16 + lane][kb] = l;
    }
  }
  __syncthreads();
  if (!values) return;
  const int l31 = lane & 31, h = lane >> 5;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = (pr + t) * 32 + l31, qi = qb * R + row;
    if (qi >= nq) continue;
    const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(s_max[0][row]);
    const float l = (l4[0] + l4[1]) + (l4[2] + l4[3]);
    const float inv = 1.f / l;
    const size_t unit = (size_t)plan.seg_unit0[seg] + (size_t)ch * nq + qi;
    // o[e][t][4 i + j]: column pw * 64 + (i / 2) * 32 + ((i & 1) * 2 + h) * 8 + (e ^ i / 2) * 4 + j
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int f = i >> 1, col = pw * 64 + f * 32 + ((i & 1) * 2 + h) * 8;
      f32x4_t x = {o[f][t][i * 4], o[f][t][i * 4 + 1], o[f][t][i * 4 + 2], o[f][t][i * 4 + 3]};
      f32x4_t y = {o[1 - f][t][i * 4], o[1 - f][t][i * 4 + 1], o[1 - f][t][i * 4 + 2], o[1 - f][t][i * 4 + 3]};
      if (chunks == 1) {
        x *= inv; y *= inv;
        *reinterpret_cast<u32x4_t*>(a.out + ((size_t)row0 * H + qi) * DC + col) =
            (u32x4_t){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      } else {
        float* po = a.part + unit * DC + col;
        *reinterpret_cast<f32x4_t*>(po) = x;
        *reinterpret_cast<f32x4_t*>(po + 4) = y;
      }
    }
    if (chunks > 1 && pw == 0 && h == 0) {
      float* ml = a.part + (size_t)plan.units_total * DC + unit * 2;
      ml[0] = -shift_v[t]; ml[1] = l;
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
