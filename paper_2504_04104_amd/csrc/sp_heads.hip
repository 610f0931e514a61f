// Head rows on their way into the cache and back: the norms of the query and key heads, the position rotation and the cache
// append in one pass over the rows of the QKV projection; rows stored into and read from the cache as they are.  The cache holds
// float32, bf16 or 4-bit values (sp_fp4.h).
//
//   q, k : y = x * rsqrt(mean(x^2) + eps) * gain over the head's columns (where the stage has head norms), then
//          (a, b) -> (a cos - b sin, b cos + a sin) for the pairs (t, t + d_head / 2) at angle position * theta^(-2t / d_head);
//          or, by sp_stage_set_rope, the pairs (t, t + dims / 2) or (2t, 2t + 1) of the first dims columns at given frequencies, times a gain
//   v    : copied
//
// A head belongs to d_head / 8 consecutive lanes, a lane holds four pairs: columns t .. t+3 and d_head/2 + t .. + 3, or eight columns in a
// row, or columns that pass.  Sums over
// the head and maxima over the eight lanes of a 4-bit group stay in the wave; nothing goes through LDS but the angles' sines.
// Everything is float32 until the one rounding to the storage type.  Bound by the launch and a chain of lookups (request,
// its prefix, the node's depth, its page) for a tree level: one row 3.3 us, 64 rows 4.0; 640 rows, 16 MB, 6.6.
#include "sp_launch.h"
#include "sp_fp4.h"

template <typename T> __device__ __forceinline__ void load4(const T* p, float (&v)[4]);
template <> __device__ __forceinline__ void load4<float>(const float* p, float (&v)[4]) {
  const f32x4_t u = *reinterpret_cast<const f32x4_t*>(p);
  v[0] = u[0]; v[1] = u[1]; v[2] = u[2]; v[3] = u[3];
}
template <> __device__ __forceinline__ void load4<bf16_t>(const bf16_t* p, float (&v)[4]) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<f32x4_t*>(p) = (f32x4_t){v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store4(bf16_t* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// Columns ca .. ca+3 and cb .. cb+3 of a head into slot `slot` of a plane of the cache (all lanes of the wave that have a head
// come here together: the groups' maxima are taken across lanes; eight lanes have 32 columns in a row twice).
template <typename T, bool FP4>
__device__ __forceinline__ void put_row(const KvGeom& g, size_t plane, size_t slot, int ca, int cb, const float (&a)[4], const float (&b)[4]) {
  char* row = g.kv + plane * g.plane_bytes + slot * g.row_bytes;
  if constexpr (!FP4) {
    store4(reinterpret_cast<T*>(row) + ca, a);
    store4(reinterpret_cast<T*>(row) + cb, b);
  } else {
    // four values of eight lanes are a group, in either half
    float ma = 0.f, mb = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { ma = fmaxf(ma, fabsf(a[i])); mb = fmaxf(mb, fabsf(b[i])); }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) { ma = fmaxf(ma, __shfl_xor(ma, o, 64)); mb = fmaxf(mb, __shfl_xor(mb, o, 64)); }
    const uint32_t ba = fp4_biased(ma), bb = fp4_biased(mb);
    reinterpret_cast<unsigned short*>(row)[ca >> 2] = (unsigned short)fp4_codes4(a, fp4_scale(ba));
    reinterpret_cast<unsigned short*>(row)[cb >> 2] = (unsigned short)fp4_codes4(b, fp4_scale(bb));
    if ((ca & 31) == 0) {
      unsigned char* sc = reinterpret_cast<unsigned char*>(g.scales + plane * g.scale_plane_bytes + slot * 4);
      sc[ca / FP4_GROUP] = (unsigned char)ba;
      sc[cb / FP4_GROUP] = (unsigned char)bb;
    }
  }
}

struct AppendArgs {
  const void* x;            // PART: float32 [S][rows][(n_q + 2 n_kv) * d_head], else the storage type, one slice
  int S;
  size_t part_stride;
  const RowInfo* rows;      // PART: the call's row descriptors and rotary tables ([rows][d_head], cosines first)
  const float* cs;
  const ReqMeta* meta;      // else: they are formed here
  const ReqTables* tables;
  double log2_theta;
  const void* gain_q;       // [d_head], null: no norms
  const void* gain_k;
  float eps;
  void* q;                  // [rows][n_q * d_head]
  KvGeom g;
  int layer, n_q, n_kv, d_head;
};
// A rotation of the stage's own (SET; PART: its layout and dims, the angles are in cs), or none beside the config's.
struct NoRope {};
template <bool SET> struct RopeArg { typedef NoRope type; };
template <> struct RopeArg<true> { typedef StageRope type; };

// grid: (rows, ceil(heads / (256 / (d_head / 8)))).  T: storage of the rows, and of the cache unless FP4.  The rotation that a stage
// is created with has kernels of its own: in one with the others, which look up layout, columns and frequencies, one row takes 4.1 us in place
// of 3.3, 64 rows 4.6 and 4.0, 640 rows 7.0 and 6.6.
template <typename T, bool FP4, bool PART, bool SET>
__global__ void __launch_bounds__(256) k_head_append(AppendArgs a, FwdBatch b, typename RopeArg<SET>::type rope) {
  __shared__ float s_cs[128];
  const int half = a.d_head >> 1, tph = half >> 2, row = blockIdx.x;
  const int head = blockIdx.y * (256 / tph) + threadIdx.x / tph;
  const int t = (threadIdx.x % tph) * 4;
  // The lane's columns: in halves four pairs of the rotated columns, or, behind their lanes, columns that pass; interleaved two
  // pairs and two pairs.
  int pairs = half, dims = a.d_head;
  bool halves = true;
  if constexpr (SET) { dims = rope.dims; pairs = dims >> 1; halves = rope.layout == 0; }
  const bool passes = SET && halves && t >= pairs;
  const int ca = passes ? dims + t - pairs : t, cb = !halves ? half + t : passes ? dims + half - pairs + t - pairs : pairs + t;
  const int heads = a.n_q + 2 * a.n_kv;
  const bool on = head < heads, rotated = head < a.n_q + a.n_kv;

  // the row's values are asked for before the position is known
  float u[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (on) {
    const size_t at = ((size_t)row * heads + head) * a.d_head;
    if constexpr (PART) {
      const float* p = reinterpret_cast<const float*>(a.x) + at;
      for (int s = 0; s < a.S; ++s) {
        float du[4], dv[4];
        load4(p + (size_t)s * a.part_stride + ca, du);
        load4(p + (size_t)s * a.part_stride + cb, dv);
#pragma unroll
        for (int i = 0; i < 4; ++i) { u[i] += du[i]; v[i] += dv[i]; }
      }
    } else {
      load4(reinterpret_cast<const T*>(a.x) + at + ca, u);
      load4(reinterpret_cast<const T*>(a.x) + at + cb, v);
    }
  }
  const bool normed = a.gain_q != nullptr && rotated;
  float gu[4] = {1.f, 1.f, 1.f, 1.f}, gv[4] = {1.f, 1.f, 1.f, 1.f};
  if (normed) {
    const T* gain = reinterpret_cast<const T*>(head < a.n_q ? a.gain_q : a.gain_k);
    load4(gain + ca, gu);
    load4(gain + cb, gv);
  }

  size_t slot;
  const float* cs;
  if constexpr (PART) {
    const RowInfo ri = a.rows[row];
    slot = sp_phys_slot(a.g, ri.req, ri.base, ri.P + ri.node);
    cs = a.cs + (size_t)row * a.d_head;
  } else {
    // Few requests one after the other, many a lane each (640 rows of 32 requests 10.0 us one after the other, 6.8; one request 3.6
    // and, a lane each, 3.9).
    static_assert(SP_BATCH <= 64, "a lane per request");
    const int lane = threadIdx.x & 63;
    int seg = 0;
    if (b.n_req > 4) seg = __popcll(__builtin_amdgcn_ballot_w64(lane < b.n_req && row >= b.row0[lane])) - 1;
    else while (seg + 1 < b.n_req && row >= b.row0[seg + 1]) ++seg;
    const int req = b.req[seg], node = b.first[seg] + (row - b.row0[seg]);
    const ReqMeta m = a.meta[req];
    const int depth = a.tables[req].depth[node];
    slot = sp_phys_slot(a.g, req, m.base, m.P + node);
    // The angle in double precision, whole turns taken off there: positions of tens of thousands keep full float accuracy.
    if ((int)threadIdx.x < pairs) {
      const double pos = (double)(m.P + depth);
      double freq;
      float gain = 1.f;
      if constexpr (SET) { freq = rope.freq[threadIdx.x]; gain = rope.gain; }
      else freq = exp2(-(2.0 * (double)threadIdx.x / (double)a.d_head) * a.log2_theta);
      const double turns = pos * freq * 0.15915494309189535;
      const float ang = (float)((turns - rint(turns)) * 6.283185307179586);
      s_cs[threadIdx.x] = cosf(ang) * gain;
      s_cs[half + threadIdx.x] = sinf(ang) * gain;
    }
    __syncthreads();
    cs = s_cs;
  }

  if (a.gain_q != nullptr) {                        // (uniform; the lanes of a head take the same way below)
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) ss += u[i] * u[i] + v[i] * v[i];
    for (int o = 1; o < tph; o <<= 1) ss += __shfl_xor(ss, o, 64);
    const float r = normed ? rsqrtf(ss / (float)a.d_head + a.eps) : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { u[i] *= r * gu[i]; v[i] *= r * gv[i]; }
  }
  if (rotated && halves && !passes) {
    float co[4], si[4];
    load4(cs + t, co);
    load4(cs + half + t, si);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = u[i], y = v[i];
      u[i] = x * co[i] - y * si[i];
      v[i] = y * co[i] + x * si[i];
    }
  } else if (rotated && !halves) {
    // (dims is a multiple of 8: four columns turn or pass together.  By a cosine of 1 and a sine of 0 what is not finite would reach
    // the column beside it)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float ua = u[2 * i], ub = u[2 * i + 1], va = v[2 * i], vb = v[2 * i + 1];
      if (ca < dims) {
        const float co = cs[ca / 2 + i], si = cs[half + ca / 2 + i];
        u[2 * i] = ua * co - ub * si;
        u[2 * i + 1] = ub * co + ua * si;
      }
      if (cb < dims) {
        const float co = cs[cb / 2 + i], si = cs[half + cb / 2 + i];
        v[2 * i] = va * co - vb * si;
        v[2 * i + 1] = vb * co + va * si;
      }
    }
  }
  if (!on) return;
  if (head < a.n_q) {
    T* dst = reinterpret_cast<T*>(a.q) + ((size_t)row * a.n_q + head) * a.d_head;
    store4(dst + ca, u);
    store4(dst + cb, v);
  } else {
    const bool is_v = head >= a.n_q + a.n_kv;
    const size_t plane = (size_t)(a.layer * 2 + (is_v ? 1 : 0)) * a.n_kv + (head - a.n_q - (is_v ? a.n_kv : 0));
    put_row<T, FP4>(a.g, plane, slot, ca, cb, u, v);
  }
}

// Rows [n][n_kv][d_head] of a request's logical slots first .. first + n - 1 into the cache (STORE) or out of it.  grid: (n, ceil(2 * n_kv * tph / 256))
template <typename T, bool FP4, bool STORE>
__global__ void __launch_bounds__(256) k_head_rows(KvGeom g, int req, long long base, int layer, int first, T* k, T* v, int n_kv, int d_head) {
  const int half = d_head >> 1, tph = half >> 2;
  const int head = blockIdx.y * (256 / tph) + threadIdx.x / tph;     // keys, then values
  if (head >= 2 * n_kv) return;
  const int t = (threadIdx.x % tph) * 4;
  const size_t row = blockIdx.x, slot = sp_phys_slot(g, req, base, first + (int)row);
  const bool is_v = head >= n_kv;
  const int h = is_v ? head - n_kv : head;
  const size_t plane = (size_t)(layer * 2 + (is_v ? 1 : 0)) * n_kv + h;
  T* p = (is_v ? v : k) + (row * n_kv + h) * d_head;
  float a[4], b[4];
  if constexpr (STORE) {
    load4(p + t, a);
    load4(p + half + t, b);
    put_row<T, FP4>(g, plane, slot, t, half + t, a, b);
  } else {
    const char* src = g.kv + plane * g.plane_bytes + slot * g.row_bytes;
    if constexpr (FP4) {
      const unsigned char* sc = reinterpret_cast<const unsigned char*>(g.scales + plane * g.scale_plane_bytes + slot * 4);
      const u32x4_t x = fp4_to_bf16x8(reinterpret_cast<const unsigned short*>(src)[t >> 2], fp4_scale(sc[t / FP4_GROUP]));
      const u32x4_t y = fp4_to_bf16x8(reinterpret_cast<const unsigned short*>(src)[(half + t) >> 2], fp4_scale(sc[(half + t) / FP4_GROUP]));
      *reinterpret_cast<uint2*>(p + t) = uint2{x.x, x.y};            // (T is bf16)
      *reinterpret_cast<uint2*>(p + half + t) = uint2{y.x, y.y};
    } else {
      load4(reinterpret_cast<const T*>(src) + t, a);
      load4(reinterpret_cast<const T*>(src) + half + t, b);
      store4(p + t, a);
      store4(p + half + t, b);
    }
  }
}

// ---- launchers -------------------------------------------------------------------
template <bool PART, bool SET>
static hipError_t go_append(int dtype, const AppendArgs& a, const FwdBatch& b, const typename RopeArg<SET>::type& rope, int M, hipStream_t st) {
  const int per = 256 / (a.d_head / 8);
  const dim3 grid(M, (a.n_q + 2 * a.n_kv + per - 1) / per), block(256);
  if (dtype == 0) hipLaunchKernelGGL((k_head_append<float, false, PART, SET>), grid, block, 0, st, a, b, rope);
  else if (a.g.scales) hipLaunchKernelGGL((k_head_append<bf16_t, true, PART, SET>), grid, block, 0, st, a, b, rope);
  else hipLaunchKernelGGL((k_head_append<bf16_t, false, PART, SET>), grid, block, 0, st, a, b, rope);
  return hipGetLastError();
}
template <bool PART>
static hipError_t go_append(int dtype, const AppendArgs& a, const FwdBatch& b, const StageRope& rope, int M, hipStream_t st) {
  return rope.on ? go_append<PART, true>(dtype, a, b, rope, M, st) : go_append<PART, false>(dtype, a, b, NoRope(), M, st);
}

static_assert(sizeof(AppendArgs) + sizeof(FwdBatch) + sizeof(StageRope) <= 4096, "kernel arguments");
hipError_t sp_launch_append_parts(int dtype, const float* part, int S, size_t part_stride, const RowInfo* rows, const float* cs,
                                  const StageRope& rope, const void* gain_q, const void* gain_k, float eps, void* qbuf, KvGeom g,
                                  int layer, int M, int n_q, int n_kv, int d_head, hipStream_t st) {
  AppendArgs a{part, S, part_stride, rows, cs, nullptr, nullptr, 0., gain_q, gain_k, eps, qbuf, g, layer, n_q, n_kv, d_head};
  FwdBatch none;
  none.n_req = 0; none.n_rows = 0;
  return go_append<true>(dtype, a, none, rope, M, st);
}
hipError_t sp_launch_append_rows(int dtype, const void* x, const FwdBatch& b, const ReqMeta* meta, const ReqTables* tables,
                                 double log2_theta, const StageRope& rope, const void* gain_q, const void* gain_k, float eps, void* q,
                                 KvGeom g, int layer, int n_q, int n_kv, int d_head, hipStream_t st) {
  AppendArgs a{x, 1, 0, nullptr, nullptr, meta, tables, log2_theta, gain_q, gain_k, eps, q, g, layer, n_q, n_kv, d_head};
  return go_append<false>(dtype, a, b, rope, b.n_rows, st);
}

template <bool STORE>
static hipError_t go_rows(int dtype, KvGeom g, int req, long long base, int layer, int first, int n, void* k, void* v, int n_kv,
                          int d_head, hipStream_t st) {
  const int per = 256 / (d_head / 8);
  const dim3 grid(n, (2 * n_kv + per - 1) / per), block(256);
  if (dtype == 0) hipLaunchKernelGGL((k_head_rows<float, false, STORE>), grid, block, 0, st, g, req, base, layer, first, (float*)k, (float*)v, n_kv, d_head);
  else if (g.scales) hipLaunchKernelGGL((k_head_rows<bf16_t, true, STORE>), grid, block, 0, st, g, req, base, layer, first, (bf16_t*)k, (bf16_t*)v, n_kv, d_head);
  else hipLaunchKernelGGL((k_head_rows<bf16_t, false, STORE>), grid, block, 0, st, g, req, base, layer, first, (bf16_t*)k, (bf16_t*)v, n_kv, d_head);
  return hipGetLastError();
}
hipError_t sp_launch_kv_store(int dtype, KvGeom g, int req, long long base, int layer, int first, int n, const void* k, const void* v,
                              int n_kv, int d_head, hipStream_t st) {
  return go_rows<true>(dtype, g, req, base, layer, first, n, const_cast<void*>(k), const_cast<void*>(v), n_kv, d_head, st);
}
hipError_t sp_launch_kv_load(int dtype, KvGeom g, int req, long long base, int layer, int first, int n, void* k, void* v, int n_kv,
                             int d_head, hipStream_t st) {
  return go_rows<false>(dtype, g, req, base, layer, first, n, k, v, n_kv, d_head, st);
}

// ---- row descriptors and plan of an attention call of its own ---------------------
__global__ void __launch_bounds__(256) k_call_rows(AttnPlan b, AttnPlan* plan_dev, const ReqMeta* meta, const ReqTables* tables, RowInfo* rows,
                                                    int M) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < M) {
    int seg = 0;                                     // (in no order of their rows)
    while (seg + 1 < b.n_seg && (r < b.seg_row0[seg] || r >= b.seg_row0[seg] + b.seg_rows[seg])) ++seg;
    const int req = b.seg_req[seg], node = b.seg_first[seg] + (r - b.seg_row0[seg]);
    const ReqMeta m = meta[req];
    RowInfo ri;
    ri.base = m.base; ri.req = req; ri.node = node; ri.pos = m.P + tables[req].depth[node]; ri.P = m.P; ri.T = m.T;
    rows[r] = ri;
  }
  if (blockIdx.x == 0) {
    const uint32_t* src = reinterpret_cast<const uint32_t*>(&b);
    uint32_t* dst = reinterpret_cast<uint32_t*>(plan_dev);
    for (int i = threadIdx.x; i < (int)(sizeof(AttnPlan) / 4); i += 256) dst[i] = src[i];
  }
}
hipError_t sp_launch_call_rows(const AttnPlan& plan, AttnPlan* plan_dev, const ReqMeta* meta, const ReqTables* tables, RowInfo* rows,
                               int M, hipStream_t st) {
  hipLaunchKernelGGL(k_call_rows, dim3((M + 255) / 256), dim3(256), 0, st, plan, plan_dev, meta, tables, rows, M);
  return hipGetLastError();
}
