// Tree attention over a cache held in 4 bits (sp_fp4.h): softmax(q K^T / sqrt(d_head) + tree mask) V per (request, query head),
// K and V as the values that the cache holds, q and the result in bf16, scores and sums in float32.
//
// Work is split as in the bf16 kernel: a workgroup owns (request, KV head, block of query rows, chunk of slots), its waves cut
// the chunk into runs of 32-slot tiles, keep an online softmax each and are folded through LDS; chunks of one range are joined
// by a second kernel.  What is different is the way of a tile.  Both operands become bf16 by one conversion instruction for two
// values, with the group's scale in it, so nothing is corrected behind the products:
//   S^T = K Q^T : the contraction's order over the head's columns is free, so that lane (slot l % 16, kg = l / 16) takes the
//                 quarter kg of a slot's row as it lies in memory: 16 bytes, of one group at d_head = 128, one scale.  A load
//                 instruction covers 1 KB in a row, and K goes from memory to the matrix cores without LDS.
//   O^T = V^T P^T: needs the slots of a column side by side: the lane converts the V bytes that it got the same way, leaves them
//                 in LDS as bf16 rows (the wave's own 32 x d_head tile) and takes them back by transposing reads.
#include "sp_attn.h"
#include "sp_fp4.h"

struct Fp4AttnArgs {
  const bf16_t* q;          // [M][n_q][DH]
  const ReqTables* tables;
  KvGeom g;
  int layer, n_q, n_kv;
  float* part_o;            // [units][DH], followed by [units][2] (running max, sum)
  bf16_t* out;              // rows of n_q * DH columns, in fragment order or (frag false) row-major
  bool frag;
  const AttnPlan* plan;     // device copy of the call's plan; unused where the plan is an argument of the launch
};
struct NoPlan { int unused; };
template <bool VAL> struct PlanArg { typedef NoPlan type; };
template <> struct PlanArg<true> { typedef AttnPlan type; };
static_assert(sizeof(Fp4AttnArgs) + sizeof(AttnPlan) <= 4096, "kernel arguments");

// Byte of column unit `u` (8 columns) of slot `row` in the wave's V tile: units are exchanged by the row's number as in the bf16
// kernel, so that sixteen rows' stores of the same unit, and the four rows x four units of a transposing read, lie in different
// units of a 256-byte line.  Heads of 64: two slots to a line.
template <int DH>
__device__ __forceinline__ int v_place(int row, int u) {
  if constexpr (DH == 128) return row * 256 + (u ^ ((row & 3) * 4 + ((row >> 2) & 3))) * 16;
  else return (row >> 1) * 256 + ((((row & 1) << 3) | u) ^ (((row >> 1) & 1) * 4 + ((row >> 2) & 3))) * 16;
}

// A tile of 32 slots in registers: for each half of 16 slots the lane's quarter of its slot's row and that row's scales.
template <int DH>
struct Fp4Tile {
  static constexpr int W = DH / 32;                // dwords of a quarter row: four groups of eight codes, or two
  uint32_t c[2][W];
  uint32_t s[2];
};

// NW waves, QT tiles of 16 query rows that every wave takes through its run, PF tiles in flight.
template <int DH, int QT, int NW, int PF, bool PAGED>
__device__ __forceinline__ void attn_fp4(const Fp4AttnArgs& a, const AttnPlan& plan) {
  constexpr int ND = DH / 16, W = DH / 32, RB = DH / 2;
  __shared__ __attribute__((aligned(16))) char s_v[NW * 32 * DH * 2];     // V tiles; later a query tile's states
  __shared__ float s_m[NW][QT * 16];
  __shared__ float s_l[NW][QT * 16];

  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, kg = lane >> 4;
  // KV head fastest: the blocks and chunks of a head share one XCD's L2
  const int item = uni(blockIdx.x / a.n_kv);
  const int kvh = blockIdx.x - item * a.n_kv;
  int seg = 0;
  const int n_seg = plan.n_seg, units_total = plan.units_total;
  if (n_seg > 1)                                   // each lane looks at a segment
    seg = uni(__popcll(__builtin_amdgcn_ballot_w64(lane < n_seg && item >= plan.seg_item0[lane])) - 1);
  const int chunks = plan.seg_chunks[seg], seg_rows = plan.seg_rows[seg], row0 = plan.seg_row0[seg];
  const int P = plan.seg_P[seg], span = P + plan.seg_T[seg], clen = plan.seg_clen[seg], req = plan.seg_req[seg];
  const int seg_first = plan.seg_first[seg], unit0 = plan.seg_unit0[seg];
  const int local = item - plan.seg_item0[seg];
  const int qb = uni(local / chunks), ch = local - qb * chunks;
  const int g = a.n_q / a.n_kv;
  const float inv_g = 1.f / (float)g;              // (qi + 0.5) * inv_g truncates to qi / g for these small integers
  const int nqrows = seg_rows * g;                 // query rows of this (request, KV head)
  const int c0 = ch * clen, c1 = min(c0 + clen, span);
  const int ntiles = (c1 - c0 + 31) >> 5;
  const int w0 = c0 + 32 * ((wave * ntiles) / NW);
  const int w1 = min(c0 + 32 * (((wave + 1) * ntiles) / NW), c1);

  const size_t base = PAGED ? 0 : (size_t)plan.seg_base[seg];
  const size_t kp = (size_t)(a.layer * 2 + 0) * a.n_kv + kvh, vp = (size_t)(a.layer * 2 + 1) * a.n_kv + kvh;
  const char* planes[2] = {a.g.kv + kp * a.g.plane_bytes + base * RB, a.g.kv + vp * a.g.plane_bytes + base * RB};
  const char* scales[2] = {a.g.scales + kp * a.g.scale_plane_bytes + base * 4, a.g.scales + vp * a.g.scale_plane_bytes + base * 4};
  typedef const __attribute__((address_space(4))) int* const_int_p;
  const const_int_p pt = PAGED ? (const_int_p)(uintptr_t)(a.g.page_table + (size_t)req * a.g.pt_stride) : nullptr;
  const int pg_sh = PAGED ? a.g.pg_shift : 0, pg_mask = (1 << pg_sh) - 1;
  // Loads of the tile with first slot s0 of the wave's run: buffers as long as the tile's rows inside the request's data, so that
  // rows behind them come back as zeros without a memory access; no rows at all behind the run.
  Fp4Tile<DH> kt[PF], vt[PF];
  auto fetch = [&](Fp4Tile<DH> (&t)[PF], int slot, int which, size_t phys, int rows) {
    const auto cb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(planes[which]) + phys * RB, (short)0, rows * RB, 0x00020000);
    const auto sb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(scales[which]) + phys * 4, (short)0, rows * 4, 0x00020000);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = h * 16 + l15;
      if constexpr (W == 4) {
        const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(cb, row * RB + kg * 16, 0, 0);
        t[slot].c[h][0] = v.x; t[slot].c[h][1] = v.y; t[slot].c[h][2] = v.z; t[slot].c[h][3] = v.w;
      } else {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(cb, row * RB + kg * 8, 0, 0);
        t[slot].c[h][0] = v[0]; t[slot].c[h][1] = v[1];
      }
      t[slot].s[h] = __builtin_amdgcn_raw_buffer_load_b32(sb, row * 4, 0, 0);
    }
  };
  auto fetch_tile = [&](int slot, int s0) {
    const int rows = s0 < w1 ? uni(min(32, span - s0)) : 0;
    const int t0 = rows > 0 ? s0 : 0;
    const size_t phys = PAGED ? ((size_t)pt[t0 >> pg_sh] << pg_sh) + (t0 & pg_mask) : (size_t)t0;
    fetch(kt, slot, 0, phys, rows);
    fetch(vt, slot, 1, phys, rows);
  };
#pragma unroll
  for (int p = 0; p < PF; ++p) fetch_tile(p, w0 + p * 32);

  // ---- query fragments and ancestor masks of this lane's query row per tile ------
  u32x4_t qf[QT][W];
  unsigned long long anc[QT][SP_W];
  const ReqTables* tab = a.tables + req;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qi = qb * (QT * 16) + t * 16 + l15;  // index inside (request, KV head): node_local * g + gq
    const bool ok = qi < nqrows;
    const int nl = ok ? (int)(((float)qi + 0.5f) * inv_g) : 0, gq = ok ? qi - nl * g : 0;
    const bf16_t* qp = a.q + ((size_t)(row0 + nl) * a.n_q + (size_t)kvh * g + gq) * DH + kg * (DH / 4);
#pragma unroll
    for (int s = 0; s < W; ++s) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(qp + s * 8);
      qf[t][s] = ok ? v : (u32x4_t){0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int w = 0; w < SP_W; ++w) {
      const unsigned long long v = tab->anc[seg_first + nl][w];
      anc[t][w] = ok ? v : 0ull;
    }
  }

  AttnState<QT, ND> st;
  st.init();
  char* vl = s_v + wave * (32 * DH * 2);
  int va[DH / 32];
#pragma unroll
  for (int G = 0; G < DH / 32; ++G) va[G] = v_place<DH>(kg * 4 + (l15 >> 2), G * 4 + (l15 & 3));
  const int group_shift = kg * (DH / 4) / FP4_GROUP * 8;             // of the lane's scale in a row's four bytes

  for (int r0 = w0; r0 < w1; r0 += 32 * PF) {
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int s0 = r0 + p * 32;
      if (s0 < w1) {
        f32x4_t sacc[QT][2];
        uint32_t pb[QT][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sc = fp4_scale((kt[p].s[h] >> group_shift) & 255u);
#pragma unroll
          for (int t = 0; t < QT; ++t) sacc[t][h] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < W; ++s) {
            const u32x4_t kf = fp4_to_bf16x8(kt[p].c[h][s], sc);
#pragma unroll
            for (int t = 0; t < QT; ++t)
              sacc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qf[t][s]),
                                                                   sacc[t][h], 0, 0, 0);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sc = fp4_scale((vt[p].s[h] >> group_shift) & 255u);
#pragma unroll
          for (int s = 0; s < W; ++s)
            *reinterpret_cast<u32x4_t*>(vl + v_place<DH>(h * 16 + l15, kg * W + s)) = fp4_to_bf16x8(vt[p].c[h][s], sc);
        }
        fetch_tile(p, s0 + 32 * PF);
        attn_softmax<QT, ND>(st, sacc, pb, anc, s0, w1, P, span, kg);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int G = 0; G < DH / 32; ++G)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint2 lo = read_transposed(vl + va[G] + e * 8), hi = read_transposed(vl + va[G] + e * 8 + 16 * DH * 2);
            const u32x4_t vf = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
            for (int t = 0; t < QT; ++t)
              st.o[t][2 * G + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf), *reinterpret_cast<const bf16x8_t*>(&pb[t][0]),
                                                                        st.o[t][2 * G + e], 0, 0, 0);
          }
        __builtin_amdgcn_wave_barrier();
      }
    }
  }

  // ---- fold the waves' states, one query tile at a time (fixed order, so results do not depend on timing) ----
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    st.lrun[t] = quad_rows_sum(st.lrun[t]);
    st.mrun[t] = st.mrun[t] * attn_scale<ND>();     // to the log2 domain (-inf stays -inf)
    if (kg == 0) s_m[wave][t * 16 + l15] = st.mrun[t];
  }
  __syncthreads();                                  // every wave is done with its V tile; maxima are posted
  f32x4_t* fold = reinterpret_cast<f32x4_t*>(s_v);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, s_m[w][t * 16 + l15]);
    const float f = (st.mrun[t] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(st.mrun[t] - m);
#pragma unroll
    for (int d = 0; d < ND; ++d) fold[(wave * ND + d) * 64 + lane] = st.o[t][d] * f;
    if (kg == 0) s_l[wave][t * 16 + l15] = st.lrun[t] * f;
    __syncthreads();
    const int qi = qb * (QT * 16) + t * 16 + l15;
    if (wave < DH / 32 && qi < nqrows) {            // one wave for 32 columns
      const int G = wave;
      f32x4_t e0 = {0.f, 0.f, 0.f, 0.f}, e1 = {0.f, 0.f, 0.f, 0.f};
      float lsum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        e0 += fold[(w * ND + 2 * G) * 64 + lane];
        e1 += fold[(w * ND + 2 * G + 1) * 64 + lane];
        lsum += s_l[w][t * 16 + l15];
      }
      // e0[i] / e1[i] are output columns G*32 + 8*kg + i and + 4 of query row t*16 + l15
      const int nl = (int)(((float)qi + 0.5f) * inv_g), head = kvh * g + qi - nl * g;
      if (chunks == 1) {
        const float inv = 1.f / lsum;
        *reinterpret_cast<u32x4_t*>(a.out + row_at(a.frag, row0 + nl, head * DH + G * 32 + 8 * kg, a.n_q * DH)) =
            (u32x4_t){pack_bf16x2(e0[0] * inv, e0[1] * inv), pack_bf16x2(e0[2] * inv, e0[3] * inv),
                      pack_bf16x2(e1[0] * inv, e1[1] * inv), pack_bf16x2(e1[2] * inv, e1[3] * inv)};
      } else {
        const size_t unit = (size_t)unit0 + (size_t)ch * seg_rows * a.n_q + (size_t)nl * a.n_q + head;
        float* po = a.part_o + unit * DH;
        *reinterpret_cast<f32x4_t*>(po + G * 32 + 8 * kg) = e0;
        *reinterpret_cast<f32x4_t*>(po + G * 32 + 8 * kg + 4) = e1;
        if (G == 0 && kg == 0) {
          float* ml = a.part_o + (size_t)units_total * DH + unit * 2;
          ml[0] = m; ml[1] = lsum;
        }
      }
    }
    if (t + 1 < QT) __syncthreads();
  }
}

template <int DH, int QT, int NW, int PF, bool PAGED, bool VAL>
__global__ void __launch_bounds__(64 * NW) k_attn_fp4(Fp4AttnArgs a, typename PlanArg<VAL>::type plan) {
  if constexpr (VAL) attn_fp4<DH, QT, NW, PF, PAGED>(a, plan);
  else attn_fp4<DH, QT, NW, PF, PAGED>(a, *a.plan);
}
template <int DH, bool VAL>
__global__ void __launch_bounds__(256) k_attn_fp4_merge(Fp4AttnArgs a, int M, typename PlanArg<VAL>::type plan) {
  if constexpr (VAL) attn_merge<DH>(plan, a.part_o, a.out, a.frag, a.n_q, M);
  else attn_merge<DH>(*a.plan, a.part_o, a.out, a.frag, a.n_q, M);
}

template <int DH, int QT, int NW, int PF>
static void go(const Fp4AttnArgs& a, const AttnPlan& plan, hipStream_t st) {
  const dim3 grid(plan.total_items * a.n_kv), block(64 * NW);
  const NoPlan none{0};
  if (a.plan) {
    if (a.g.page_table) hipLaunchKernelGGL((k_attn_fp4<DH, QT, NW, PF, true, false>), grid, block, 0, st, a, none);
    else hipLaunchKernelGGL((k_attn_fp4<DH, QT, NW, PF, false, false>), grid, block, 0, st, a, none);
  } else {
    if (a.g.page_table) hipLaunchKernelGGL((k_attn_fp4<DH, QT, NW, PF, true, true>), grid, block, 0, st, a, plan);
    else hipLaunchKernelGGL((k_attn_fp4<DH, QT, NW, PF, false, true>), grid, block, 0, st, a, plan);
  }
}
template <int DH>
static hipError_t launch(const Fp4AttnArgs& a, const AttnPlan& plan, int M, hipStream_t st) {
  switch (plan.qt) {
    case 1: go<DH, 1, 8, 4>(a, plan, st); break;
    case 2: go<DH, 2, 8, 3>(a, plan, st); break;
    case 4: go<DH, 4, 4, 2>(a, plan, st); break;
    default: return hipErrorInvalidValue;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !plan.any_split) return e;
  const dim3 grid(((M + 7) / 8 * a.n_q + 7) / 8 * 16);
  if (a.plan) hipLaunchKernelGGL((k_attn_fp4_merge<DH, false>), grid, dim3(256), 0, st, a, M, NoPlan{0});
  else hipLaunchKernelGGL((k_attn_fp4_merge<DH, true>), grid, dim3(256), 0, st, a, M, plan);
  return hipGetLastError();
}

hipError_t sp_launch_attn_fp4(const bf16_t* q, const ReqTables* tables, KvGeom g, int layer, const AttnPlan& plan,
                              const AttnPlan* plan_dev, float* part, bf16_t* out, bool frag, int M, int n_q, int n_kv, int d_head,
                              hipStream_t st) {
  if (!g.scales || g.row_bytes != d_head / 2) return hipErrorInvalidValue;
  Fp4AttnArgs a;
  a.q = q; a.tables = tables; a.g = g; a.layer = layer; a.n_q = n_q; a.n_kv = n_kv;
  a.part_o = part; a.out = out; a.frag = frag; a.plan = plan_dev;
  if (d_head == 128) return launch<128>(a, plan, M, st);
  if (d_head == 64) return launch<64>(a, plan, M, st);
  return hipErrorInvalidValue;
}
