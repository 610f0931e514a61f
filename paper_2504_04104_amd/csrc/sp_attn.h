// What the attention kernels have in common: the merge of ranges that were cut into chunks.
#pragma once
#include "sp_launch.h"

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
