// What the attention kernels have in common: the online softmax of a wave under the tree mask, the transposing reads of a V
// tile, and the merge of ranges that were cut into chunks.
#pragma once
#include "sp_launch.h"

// Online softmax of a wave over QT tiles of 16 query rows.  mrun is the running maximum of the raw scores q.k; negm =
// -mrun*sc (0 while mrun is -inf), so that exp2(fma(s, sc, negm)) is the softmax weight.
// ND: tiles of 16 columns in a head.
template <int QT, int ND = 8>
struct AttnState {
  f32x4_t o[QT][ND];
  float mrun[QT], lrun[QT], negm[QT];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      mrun[t] = -INFINITY; lrun[t] = 0.f; negm[t] = 0.f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[t][d] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
  }
};
// 1 / sqrt(16 ND) * log2(e)
template <int ND>
__host__ __device__ constexpr float attn_scale() {
  static_assert(ND == 8 || ND == 4, "heads of 128 or 64 columns");
  return (ND == 8 ? 0.08838834764831845f : 0.125f) * 1.4426950408889634f;
}

// Scores of the tile with first slot s0, of a run that ends at w1, to weights (bf16 pairs, in the order of sacc's slots).
template <int QT, int ND = 8>
__device__ __forceinline__ void attn_softmax(AttnState<QT, ND>& st, const f32x4_t (&sacc)[QT][2], uint32_t (&pb)[QT][4],
                                             const unsigned long long (&anc)[QT][SP_W], int s0, int w1, int P, int span, int kg) {
  constexpr float sc = attn_scale<ND>();
  const bool tail = s0 + 32 > P || s0 + 32 > w1;   // tile touches the tree region or the run's end
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float sv[8];
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
      for (int i = 0; i < 4; ++i) sv[t2 * 4 + i] = sacc[t][t2][i];
    if (tail) {
      // bits [n0, n0+64) of the row's 256-bit ancestor mask, n0 = first tree index of the tile
      const int n0 = s0 - P;
      unsigned long long win = 0ull;
#pragma unroll
      for (int w = 0; w < SP_W; ++w) {
        const int sh = w * 64 - n0;
        if (sh > -64 && sh < 64) win |= sh >= 0 ? (anc[t][w] << sh) : (anc[t][w] >> (-sh));
      }
      const int lim = w1 - s0, pfx = P - s0, tl = span - s0;   // offsets below: in run / committed / live
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int off = (j >> 2) * 16 + kg * 4 + (j & 3);
        const bool vis = (off < lim) & ((off < pfx) | ((off < tl) & (bool)((win >> off) & 1ull)));
        sv[j] = vis ? sv[j] : -INFINITY;
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
    // The running maximum only has to bound the scores, so it is raised (and the
    // accumulators rescaled) only when some lane of the wave sees a larger score.
    if (__builtin_amdgcn_ballot_w64(mx > st.mrun[t])) {
      mx = quad_rows_max(mx);
      const float mnew = fmaxf(st.mrun[t], mx);
      const float alpha = (mnew == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f((st.mrun[t] - mnew) * sc);  // 0 from -inf
      st.lrun[t] *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) st.o[t][d] *= alpha;
      st.mrun[t] = mnew;
      st.negm[t] = (mnew == -INFINITY) ? 0.f : -mnew * sc;
    }
    float pv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) pv[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[j], sc, st.negm[t]));
    st.lrun[t] += ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
#pragma unroll
    for (int j = 0; j < 4; ++j) pb[t][j] = pack_bf16x2(pv[2 * j], pv[2 * j + 1]);
  }

}

// Sixteen lanes read four slots x 16 columns, lane 4c + x of them gets the four slots of one column.
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
__device__ __forceinline__ uint2 read_transposed(const char* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p)));
#else
  return uint2{0u, 0u};
#endif
}
// One wave per (row, query head) of the requests that were cut into several chunks: combine the
// chunk partials (log2-domain maxima).  Lane c first takes chunk c's (max, sum) and turns them into
// the chunk's weight; the outputs are then accumulated chunk by chunk, two columns per lane.
// (a workgroup of 256 threads; part_o: [units][DH], followed by [units][2]; out: rows of n_q * DH columns)
template <int DH>
__device__ __forceinline__ void attn_merge(const AttnPlan& plan, const float* part_o, bf16_t* out, bool frag, int n_q, int M) {
  static_assert(DH == 128 || DH == 64, "one or two columns per lane");
  int sg_chunks = plan.seg_chunks[0], sg_rows = plan.seg_rows[0], sg_unit0 = plan.seg_unit0[0], sg_row0 = plan.seg_row0[0];
  const int n_seg = plan.n_seg;
  const float* part_ml = part_o + (size_t)plan.units_total * DH;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // a workgroup takes four rows of a head; the two that fill the output's 128-byte lines (eight rows in fragment order)
  // run on the same XCD, whose L2 puts the lines together
  const int pair = (blockIdx.x >> 4) * 8 + (blockIdx.x & 7), row8 = pair / n_q, head = pair - row8 * n_q;
  const int row = row8 * 8 + ((blockIdx.x >> 3) & 1) * 4 + wave;
  if (row >= M) return;
  if (n_seg > 1) {                       // each lane looks at a segment
    const int first = plan.seg_row0[lane], seg = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(lane < n_seg && row >= first && row < first + plan.seg_rows[lane])) - 1;
    sg_chunks = plan.seg_chunks[seg]; sg_rows = plan.seg_rows[seg]; sg_unit0 = plan.seg_unit0[seg]; sg_row0 = plan.seg_row0[seg];
  }
  const int chunks = sg_chunks, seg_rows = sg_rows;
  if (chunks == 1) return;               // written directly by the attention kernel
  const size_t stride = (size_t)seg_rows * n_q;
  const size_t u0 = (size_t)sg_unit0 + (size_t)(row - sg_row0) * n_q + head;
  // the lane's columns of a partial row
  auto piece = [&](const float* po) -> float2 {
    if constexpr (DH == 128) return *reinterpret_cast<const float2*>(po + 2 * lane);
    else return float2{po[lane], 0.f};
  };
  float acc0 = 0.f, acc1 = 0.f, lsum = 0.f, mx = -INFINITY;
  for (int c0 = 0; c0 < chunks; c0 += 64) {        // blocks of 64 chunks (one is the rule)
    const int c = c0 + lane;
    float m = -INFINITY, l = 0.f;
    if (c < chunks) {
      const float2 ml = *reinterpret_cast<const float2*>(part_ml + (u0 + c * stride) * 2);
      m = ml.x; l = ml.y;
    }
    const float bm = wave_max(m);
    const float nmx = fmaxf(mx, bm);
    if (nmx == -INFINITY) continue;
    const float resc = (mx == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(mx - nmx);
    acc0 *= resc; acc1 *= resc; lsum *= resc;
    mx = nmx;
    const float wgt = (m == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m - mx);
    lsum += wave_sum(wgt * l);
    const int nb = min(64, chunks - c0);
    int j = 0;
    // sixteen chunks' partial rows in flight at a time: the loop is a chain of memory round trips otherwise
    for (; j + 16 <= nb; j += 16) {
      float o0[16], o1[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float* po = part_o + (u0 + (size_t)(c0 + j + i) * stride) * DH;
        const float2 v = piece(po);
        o0[i] = v.x; o1[i] = v.y;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w1 = __shfl(wgt, j + i, 64);
        acc0 += w1 * o0[i]; acc1 += w1 * o1[i];
      }
    }
    for (; j + 4 <= nb; j += 4) {
      float w4[4], o0[4], o1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w4[i] = __shfl(wgt, j + i, 64);
        const float* po = part_o + (u0 + (size_t)(c0 + j + i) * stride) * DH;
        const float2 v = piece(po);
        o0[i] = v.x; o1[i] = v.y;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) { acc0 += w4[i] * o0[i]; acc1 += w4[i] * o1[i]; }
    }
    for (; j < nb; ++j) {
      const float w1 = __shfl(wgt, j, 64);
      const float2 v = piece(part_o + (u0 + (size_t)(c0 + j) * stride) * DH);
      acc0 += w1 * v.x; acc1 += w1 * v.y;
    }
  }
  const float inv = 1.f / lsum;
  if constexpr (DH == 128)
    *reinterpret_cast<uint32_t*>(out + row_at(frag, row, head * DH + 2 * lane, n_q * DH)) = pack_bf16x2(acc0 * inv, acc1 * inv);
  else
    out[row_at(frag, row, head * DH + lane, n_q * DH)] = f32_to_bf16(acc0 * inv);
}
