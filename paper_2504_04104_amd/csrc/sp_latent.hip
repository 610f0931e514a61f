// Rows of a latent cache: the append (norm of the latent, rotation of the key part that all heads share and of the query heads'
// parts, the row into its slot), rows stored and loaded as they are.
//
//   latent : c * rsqrt(mean(c^2) + eps) * gain (where the stage has norms), key part and queries: rotated at prefix_len + depth
//
// Float32 until the one rounding to bf16; the angles in double precision, whole turns taken off there.  The append is bound by its launch and
// by the chain request -> node -> depth, slot, page: one row of 16 heads 3.6 us; 668 rows of 64 heads, 12 MB in and out, 5.7.
#include "sp_launch.h"

__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const u32x4_t u = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(u[i]); v[2 * i + 1] = bf16_hi(u[i]); }
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4_t*>(p) = (u32x4_t){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// Four pairs of a rotated part, by number t .. t+3: in halves columns t .. and pairs + t .., interleaved columns 2t .. 2t + 7.  Lanes
// behind the pairs have eight columns that pass.
struct Turn { int ca, cb, t; bool turns; };
__device__ __forceinline__ Turn turn_of(int lane, int cols, const StageRope& r) {
  const int pairs = r.dims >> 1, t = lane * 4;
  Turn o;
  o.t = t;
  o.turns = t < pairs;
  if (r.layout == 0 && o.turns) { o.ca = t; o.cb = pairs + t; }
  else { o.ca = 2 * t; o.cb = 2 * t + 4; }           // (interleaved, or passing: eight columns in a row, cols of them in all)
  return o;
}
__device__ __forceinline__ void load4(const bf16_t* p, float* v) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
}
__device__ __forceinline__ void store4(bf16_t* p, const float* v) { *reinterpret_cast<uint2*>(p) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }
__device__ __forceinline__ void turn(const Turn& o, int layout, const float* s_cos, const float* s_sin, float (&v)[8]) {
  if (!o.turns) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float co = s_cos[o.t + e], si = s_sin[o.t + e];
    float& a = layout == 0 ? v[e] : v[2 * e];
    float& b = layout == 0 ? v[4 + e] : v[2 * e + 1];
    const float p = a, q = b;
    a = p * co - q * si;
    b = q * co + p * si;
  }
}

// grid: (rows, 1 + workgroups of the query heads).  blockIdx.y == 0: the row of the cache, its latent by the first wave, its key part by
// the second; else 256 / (d_rope / 8) query heads.
__global__ void __launch_bounds__(256) k_latent_append(LatentAppendArgs a, FwdBatch b) {
  __shared__ float s_cos[SP_ROPE_PAIRS], s_sin[SP_ROPE_PAIRS];
  const int row = blockIdx.x, R = a.d.d_rope, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool cache = blockIdx.y == 0;
  const int tph = R >> 3;                           // lanes of a rotated part
  const int head = ((int)blockIdx.y - 1) * (256 / tph) + (int)threadIdx.x / tph;
  const Turn o = turn_of(cache ? lane : (int)threadIdx.x % tph, R, a.rope);
  const bool part = cache ? wave == 1 && lane < tph : (int)threadIdx.x / tph < 256 / tph && head < a.d.n_heads;
  const bf16_t* src = cache ? a.kv + row * a.kv_row + a.d.d_latent : a.q + row * a.q_row + head * a.q_head;
  float v[8];
  if (part) { load4(src + o.ca, v); load4(src + o.cb, v + 4); }

  int seg = 0;
  if (b.n_req > 4) seg = __popcll(__builtin_amdgcn_ballot_w64(lane < b.n_req && row >= b.row0[lane])) - 1;
  else while (seg + 1 < b.n_req && row >= b.row0[seg + 1]) ++seg;
  const int req = b.req[seg], node = b.first[seg] + (row - b.row0[seg]);
  const ReqMeta m = a.meta[req];
  const int depth = a.tables[req].depth[node];
  if ((int)threadIdx.x < a.rope.dims >> 1) {
    const double pos = (double)(m.P + depth);
    const double turns = pos * (a.rope.on ? a.rope.freq[threadIdx.x] : exp2(-(2.0 * (double)threadIdx.x / (double)R) * a.log2_theta)) * 0.15915494309189535;
    const float ang = (float)((turns - rint(turns)) * 6.283185307179586);
    s_cos[threadIdx.x] = cosf(ang) * a.rope.gain;
    s_sin[threadIdx.x] = sinf(ang) * a.rope.gain;
  }
  __syncthreads();
  if (part) turn(o, a.rope.layout, s_cos, s_sin, v);
  if (!cache) {
    if (!part) return;
    bf16_t* dst = a.q_out + row * a.out_row + head * a.out_head;
    store4(dst + o.ca, v);
    store4(dst + o.cb, v + 4);
    return;
  }
  bf16_t* slot = reinterpret_cast<bf16_t*>(a.g.kv + (size_t)a.layer * a.g.plane_bytes + sp_phys_slot(a.g, req, m.base, m.P + node) * a.g.row_bytes);
  if (part) {
    store4(slot + a.d.d_latent + o.ca, v);
    store4(slot + a.d.d_latent + o.cb, v + 4);
  }
  if (wave != 0) return;
  // the latent: eight columns a lane, in passes of 512
  const bf16_t* c = a.kv + row * a.kv_row;
  float ss = 0.f;
  if (a.gain) {
    for (int i = lane * 8; i < a.d.d_latent; i += 512) {
      float x[8];
      load8(c + i, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
    }
    ss = wave_sum(ss);
  }
  const float r = a.gain ? rsqrtf(ss / (float)a.d.d_latent + a.eps) : 1.f;
  for (int i = lane * 8; i < a.d.d_latent; i += 512) {
    float x[8], g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    load8(c + i, x);
    if (a.gain) load8(a.gain + i, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r * g[e];
    store8(slot + i, x);
  }
}

static_assert(sizeof(LatentAppendArgs) + sizeof(FwdBatch) <= 4096, "kernel arguments");
hipError_t sp_launch_latent_append(const LatentAppendArgs& a, const FwdBatch& b, hipStream_t st) {
  const int per = 256 / (a.d.d_rope >> 3);
  hipLaunchKernelGGL(k_latent_append, dim3(b.n_rows, 1 + (a.d.n_heads + per - 1) / per), dim3(256), 0, st, a, b);
  return hipGetLastError();
}

// Rows of row_bytes, a thread a piece of 16.  One row 1.5 us; 4096 of 1152 bytes, in or out, 3.3; 32768, 75 MB read and written, 12.
template <bool STORE>
__global__ void __launch_bounds__(256) k_latent_rows(KvGeom g, int req, long long base, int layer, int first, long long units, char* rows) {
  const int per = g.row_bytes >> 4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < units; i += (long long)gridDim.x * 256) {
    const int row = (int)(i / per), u = (int)(i - (long long)row * per);
    u32x4_t* slot = reinterpret_cast<u32x4_t*>(g.kv + (size_t)layer * g.plane_bytes + sp_phys_slot(g, req, base, first + row) * g.row_bytes) + u;
    u32x4_t* mine = reinterpret_cast<u32x4_t*>(rows) + i;
    if constexpr (STORE) *slot = *mine;
    else *mine = *slot;
  }
}
hipError_t sp_launch_latent_rows(bool store, KvGeom g, int req, long long base, int layer, int first, int n, void* rows, hipStream_t st) {
  const long long units = (long long)n * (g.row_bytes >> 4), blocks = (units + 255) / 256;
  const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
  if (store) hipLaunchKernelGGL(k_latent_rows<true>, grid, dim3(256), 0, st, g, req, base, layer, first, units, (char*)rows);
  else hipLaunchKernelGGL(k_latent_rows<false>, grid, dim3(256), 0, st, g, req, base, layer, first, units, (char*)rows);
  return hipGetLastError();
}

// ---- tree attention, plain ----------------------------------------------------------
// A workgroup has a (row, head): 256 slots at a time, a score a thread, then the weights meet the latents, columns over the threads.
// (What the matrix-core kernel does not cover, and SP_FLAG_SIMPLE_KERNELS.  Each (row, head) reads the range for itself: 16 rows behind 512
// slots 189 us, 80 behind 32749 11.6 ms.)
#define LATENT_MAX 1024            // columns of a latent
__global__ void __launch_bounds__(256) k_latent_attn_simple(LatentAttnArgs a, AttnPlan plan) {
  __shared__ float s_q[LATENT_MAX + 2 * SP_ROPE_PAIRS], s_p[256], s_red[4];
  __shared__ size_t s_at[256];
  const int row = blockIdx.x, head = blockIdx.y, C = a.d.d_latent, D = C + a.d.d_rope;
  int seg = 0;
  while (seg + 1 < plan.n_seg && (row < plan.seg_row0[seg] || row >= plan.seg_row0[seg] + plan.seg_rows[seg])) ++seg;
  const int req = plan.seg_req[seg], node = plan.seg_first[seg] + row - plan.seg_row0[seg], P = plan.seg_P[seg], span = P + plan.seg_T[seg];
  const long long base = plan.seg_base[seg];
  const bf16_t* q = a.q + ((size_t)row * a.d.n_heads + head) * D;
  for (int i = threadIdx.x; i < D; i += 256) s_q[i] = bf16_to_f32(q[i]) * a.scale;
  const char* plane = a.g.kv + (size_t)a.layer * a.g.plane_bytes;
  const int wave = threadIdx.x >> 6;
  float mx = -INFINITY, l = 0.f, o[LATENT_MAX / 256];
#pragma unroll
  for (int k = 0; k < LATENT_MAX / 256; ++k) o[k] = 0.f;
  __syncthreads();
  for (int s0 = 0; s0 < span; s0 += 256) {
    const int s = s0 + threadIdx.x, j = s - P, n = min(256, span - s0);
    const bool seen = s < P || (s < span && ((a.tables[req].anc[node][j >> 6] >> (j & 63)) & 1ull));
    float sc = -INFINITY;
    if (s < span) s_at[threadIdx.x] = sp_phys_slot(a.g, req, a.g.page_table ? 0 : base, s) * a.g.row_bytes;
    if (seen) {
      const bf16_t* k = reinterpret_cast<const bf16_t*>(plane + s_at[threadIdx.x]);
      sc = 0.f;
      for (int i = 0; i < D; i += 8) {
        float x[8];
        load8(k + i, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc += s_q[i + e] * x[e];
      }
    }
    const float m = wave_max(sc);
    if ((threadIdx.x & 63) == 0) s_red[wave] = m;
    __syncthreads();
    const float mn = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), mx);
    // (minus infinity is a weight of zero also where there is nothing else yet, whose largest score it then is)
    const float corr = mx == -INFINITY ? 0.f : __expf(mx - mn), p = sc == -INFINITY ? 0.f : __expf(sc - mn);
    mx = mn;
    s_p[threadIdx.x] = p;
    l = l * corr + p;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < LATENT_MAX / 256; ++k) {
      const int col = k * 256 + threadIdx.x;
      if (col >= C) continue;
      float acc = o[k] * corr;
      // (a slot that nobody sees, or whose score is minus infinity, may hold anything)
      for (int i = 0; i < n; ++i)
        if (s_p[i] != 0.f) acc += s_p[i] * bf16_to_f32(reinterpret_cast<const bf16_t*>(plane + s_at[i])[col]);
      o[k] = acc;
    }
    __syncthreads();
  }
  const float lw = wave_sum(l);
  if ((threadIdx.x & 63) == 0) s_red[wave] = lw;
  __syncthreads();
  const float inv = 1.f / (s_red[0] + s_red[1] + s_red[2] + s_red[3]);
  bf16_t* out = a.out + ((size_t)row * a.d.n_heads + head) * C;
#pragma unroll
  for (int k = 0; k < LATENT_MAX / 256; ++k)
    if (k * 256 + (int)threadIdx.x < C) out[k * 256 + threadIdx.x] = f32_to_bf16(o[k] * inv);
}
static_assert(sizeof(LatentAttnArgs) + sizeof(AttnPlan) <= 4096, "kernel arguments");
hipError_t sp_launch_latent_attn_simple(const LatentAttnArgs& a, const AttnPlan& plan, int M, hipStream_t st) {
  if (a.d.d_latent > LATENT_MAX || a.d.d_rope > 2 * SP_ROPE_PAIRS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_latent_attn_simple, dim3(M, a.d.n_heads), dim3(256), 0, st, a, plan);
  return hipGetLastError();
}
