// Products of bf16 rows with a matrix of 4-bit weights (sp_fp4.h): out[m][n] = sum_k X[m][k] W[n][k], W as the values that its
// codes and scales stand for, sums in float32.
//
// Weights lie in units of 16 rows x 256 columns, 2176 bytes in a row of memory: twice 64 x 16 bytes of codes, lane l of a wave
// taking row l % 16 and the 32 columns (l / 16) * 32 .. of either half -- one group, one scale -- and 64 x 2 bytes of scales.
// The units of 16 rows follow each other over the columns.  Which column of X a product's operand holds is free as long as
// both sides agree: the four steps over a half take columns kg * 32 + j * 8 .. + 7 in lane kg.
//
// A workgroup of eight waves owns NS strips of 16 weight rows and MT tiles of 16 rows of X, its waves cut the columns among
// them, and their sums are added through LDS.  A conversion instruction makes two codes and their scale two bf16 values.
#include "sp_launch.h"
#include "sp_fp4.h"

#define UNIT_K 256
#define UNIT_BYTES 2176
#define GW 8                 // waves per workgroup

enum { OUT_PARTS, OUT_ROWS, OUT_GATED };

struct Fp4GemmArgs {
  const bf16_t* X;
  const char* W;
  void* out;                 // OUT_PARTS: float32 [S][M][N]; OUT_ROWS: bf16 [M][N]; OUT_GATED: bf16 [M][N / 2]
  int M, N, K, units, S;
  int groups, row_blocks;    // of strips (OUT_GATED: of pairs of strips); of 16 * MT rows
  bool frag_out;             // OUT_GATED: the rows' order
};

__device__ __forceinline__ float silu(float x) { return x / (1.f + __expf(-x)); }

// NS: strips of a workgroup; OUT_GATED: half of them gate rows, the others the up rows that belong to them.
template <int MT, int NS, int OUT, bool XFRAG, bool NT>
__global__ void __launch_bounds__(64 * GW) k_fp4_gemm(Fp4GemmArgs a) {
  constexpr int PF = NS >= 4 ? 2 : 4;              // units in flight per strip and wave
  __shared__ f32x4_t s_sum[GW][MT * NS][64];
  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63, l15 = lane & 15, kg = lane >> 4;
  // the row blocks of a group of strips on one XCD, one after the other
  const int id = blockIdx.x, xcd = id & 7, local = id >> 3;
  const int rb = uni(local % a.row_blocks), sg = uni((local / a.row_blocks) * 8 + xcd);
  const int slice = uni(sg / a.groups), group = sg - slice * a.groups;
  if (slice >= a.S) return;
  const int row0 = rb * 16 * MT, rows = min(a.M - row0, 16 * MT);
  const int strips = a.N >> 4;
  int strip[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i)
    strip[i] = OUT == OUT_GATED ? (i < NS / 2 ? group * (NS / 2) + i : (strips >> 1) + group * (NS / 2) + i - NS / 2) : group * NS + i;
  auto there = [&](int i) { return OUT == OUT_GATED ? group * (NS / 2) + (i < NS / 2 ? i : i - NS / 2) < (strips >> 1) : strip[i] < strips; };
  const int su0 = (int)((long long)slice * a.units / a.S), su1 = (int)((long long)(slice + 1) * a.units / a.S);
  const int u0 = su0 + (su1 - su0) * wave / GW, u1 = su0 + (su1 - su0) * (wave + 1) / GW;

  // buffers: loads past the run, past the strips and past the rows return zeros without a memory access (what is to be checked
  // is in the lane's offset: a scalar one is not part of the check)
  const int xrows = XFRAG ? (rows + 15) & ~15 : rows;
  const auto xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(a.X) + (size_t)row0 * a.K, (short)0, uni(xrows * a.K * 2), 0x00020000);
  const int x_lane = XFRAG ? kg * 1024 + l15 * 16 : l15 * a.K * 2 + kg * 64;
  const int x_tile = 16 * a.K * 2;

  u32x4_t wq[PF][NS][2];
  uint32_t wsc[PF][NS];
  auto fetch = [&](int p, int u) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const bool on = u < u1 && there(i);
      const auto wb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.W) + ((size_t)(on ? strip[i] : 0) * a.units + (on ? u : 0)) * UNIT_BYTES,
                                                        (short)0, on ? UNIT_BYTES : 0, 0x00020000);
#pragma unroll
      for (int b = 0; b < 2; ++b) wq[p][i][b] = __builtin_amdgcn_raw_buffer_load_b128(wb, lane * 16, b * 1024, NT ? 2 : 0);
      wsc[p][i] = __builtin_amdgcn_raw_buffer_load_b16(wb, lane * 2, 2048, NT ? 2 : 0);
    }
  };
#pragma unroll
  for (int p = 0; p < PF; ++p) fetch(p, u0 + p);

  f32x4_t acc[MT][NS];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NS; ++i) acc[t][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

  for (int ub = u0; ub < u1; ub += PF) {
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int u = ub + p;
      if (u < u1) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          u32x4_t xf[MT][4];
          const int k0 = u * UNIT_K + b * 128;
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              // (columns past the end meet weights of zero; what lies behind a row may be anything)
              int off = x_lane + t * x_tile + (XFRAG ? (k0 >> 5) * 1024 : k0 * 2);
              if (!XFRAG) off = k0 + kg * 32 < a.K ? off : 0x7fffff00;
              xf[t][j] = __builtin_amdgcn_raw_buffer_load_b128(xb, off + j * (XFRAG ? 256 : 16), 0, 0);
            }
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            const float sc = fp4_scale((wsc[p][i] >> (8 * b)) & 255u);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const u32x4_t wf = fp4_to_bf16x8(wq[p][i][b][j], sc);
#pragma unroll
              for (int t = 0; t < MT; ++t)
                acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf), __builtin_bit_cast(bf16x8_t, xf[t][j]),
                                                                    acc[t][i], 0, 0, 0);
            }
          }
        }
        fetch(p, u + PF);
      }
    }
  }

#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NS; ++i) s_sum[wave][t * NS + i][lane] = acc[t][i];
  __syncthreads();
  // a lane's four sums: row t * 16 + l15 of X, weight rows kg * 4 .. + 3 of the strip
  auto total = [&](int f) {
    f32x4_t v = s_sum[0][f][lane];
#pragma unroll
    for (int w = 1; w < GW; ++w) v += s_sum[w][f][lane];
    return v;
  };
  if constexpr (OUT == OUT_GATED) {
    for (int f = wave; f < MT * (NS / 2); f += GW) {
      const int t = f / (NS / 2), i = f - t * (NS / 2), m = t * 16 + l15;
      const f32x4_t gt = total(t * NS + i), up = total(t * NS + NS / 2 + i);
      if (m >= rows || !there(i)) continue;
      const int n = strip[0] * 16 + i * 16 + kg * 4;
      *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + row_at(a.frag_out, row0 + m, n, a.N >> 1)) =
          uint2{pack_bf16x2(silu(gt[0]) * up[0], silu(gt[1]) * up[1]), pack_bf16x2(silu(gt[2]) * up[2], silu(gt[3]) * up[3])};
    }
  } else {
    for (int f = wave; f < MT * NS; f += GW) {
      const int t = f / NS, i = f - t * NS, m = t * 16 + l15;
      const f32x4_t v = total(f);
      if (m >= rows || !there(i)) continue;
      const int n = strip[0] * 16 + i * 16 + kg * 4;
      if constexpr (OUT == OUT_PARTS)
        *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + ((size_t)slice * a.M + row0 + m) * a.N + n) = v;
      else
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + (size_t)(row0 + m) * a.N + n) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  }
}

// Sums of the slices to bf16 rows: [S][M][N] -> [M][N], or (GATED) silu of the first half of the columns times the second.
template <bool GATED>
__global__ void __launch_bounds__(256) k_fp4_fold(const float* part, bf16_t* out, int S, int M, int N) {
  const int n = GATED ? N >> 1 : N;
  const size_t stride = (size_t)M * N, total = (size_t)M * n;
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < total; i += (size_t)gridDim.x * 1024) {
    const size_t m = i / n, c = i - m * n;
    const float* p = part + m * N + c;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f}, w = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < S; ++s) {
      v += *reinterpret_cast<const f32x4_t*>(p + s * stride);
      if constexpr (GATED) w += *reinterpret_cast<const f32x4_t*>(p + s * stride + n);
    }
    if constexpr (GATED)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = silu(v[j]) * w[j];
    *reinterpret_cast<uint2*>(out + i) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
}

// One wave per unit.
__global__ void __launch_bounds__(64) k_fp4_pack(const bf16_t* in, char* out, int K, int units) {
  const int lane = threadIdx.x, l15 = lane & 15, kg = lane >> 4;
  const int strip = blockIdx.x / units, u = blockIdx.x - strip * units;
  char* dst = out + (size_t)blockIdx.x * UNIT_BYTES;
  uint32_t both = 0;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int k = u * UNIT_K + b * 128 + kg * 32;
    u32x4_t codes = {0u, 0u, 0u, 0u};
    if (k < K) {
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>(in + (size_t)(strip * 16 + l15) * K + k);
      float v[32], amax = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4_t x = p[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[i * 8 + 2 * j] = bf16_lo(x[j]); v[i * 8 + 2 * j + 1] = bf16_hi(x[j]); }
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(v[i]));
      const uint32_t biased = fp4_biased(amax);
      both |= biased << (8 * b);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo[4] = {v[i * 8], v[i * 8 + 1], v[i * 8 + 2], v[i * 8 + 3]}, hi[4] = {v[i * 8 + 4], v[i * 8 + 5], v[i * 8 + 6], v[i * 8 + 7]};
        codes[i] = fp4_codes4(lo, fp4_scale(biased)) | (fp4_codes4(hi, fp4_scale(biased)) << 16);
      }
    }
    reinterpret_cast<u32x4_t*>(dst + b * 1024)[lane] = codes;
  }
  reinterpret_cast<unsigned short*>(dst + 2048)[lane] = (unsigned short)both;
}
__global__ void __launch_bounds__(64) k_fp4_unpack(const char* in, bf16_t* out, int K, int units) {
  const int lane = threadIdx.x, l15 = lane & 15, kg = lane >> 4;
  const int strip = blockIdx.x / units, u = blockIdx.x - strip * units;
  const char* src = in + (size_t)blockIdx.x * UNIT_BYTES;
  const uint32_t both = reinterpret_cast<const unsigned short*>(src + 2048)[lane];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int k = u * UNIT_K + b * 128 + kg * 32;
    if (k >= K) continue;
    const u32x4_t codes = reinterpret_cast<const u32x4_t*>(src + b * 1024)[lane];
    u32x4_t* p = reinterpret_cast<u32x4_t*>(out + (size_t)(strip * 16 + l15) * K + k);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = fp4_to_bf16x8(codes[i], fp4_scale((both >> (8 * b)) & 255u));
  }
}

// ---- launchers -------------------------------------------------------------------
size_t sp_fp4_bytes(int N, int K) { return (size_t)(N / 16) * ((K + UNIT_K - 1) / UNIT_K) * UNIT_BYTES; }
hipError_t sp_launch_fp4_pack(const void* in, void* out, int N, int K, hipStream_t st) {
  const int units = (K + UNIT_K - 1) / UNIT_K;
  hipLaunchKernelGGL(k_fp4_pack, dim3(N / 16 * units), dim3(64), 0, st, (const bf16_t*)in, (char*)out, K, units);
  return hipGetLastError();
}
hipError_t sp_launch_fp4_unpack(const void* in, void* out, int N, int K, hipStream_t st) {
  const int units = (K + UNIT_K - 1) / UNIT_K;
  hipLaunchKernelGGL(k_fp4_unpack, dim3(N / 16 * units), dim3(64), 0, st, (const char*)in, (bf16_t*)out, K, units);
  return hipGetLastError();
}

// How a product is cut: tiles of rows and strips of a workgroup, and slices of the columns where the strips leave CUs idle.
struct Fp4Split { int mt, ns, S; };
static Fp4Split split_of(int M, int N, int K, bool gated, int n_cu) {
  Fp4Split f;
  const int units = (K + UNIT_K - 1) / UNIT_K, strips = N / 16;
  f.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  const int blocks = (M + 16 * f.mt - 1) / (16 * f.mt);
  f.ns = strips * blocks >= 4 * n_cu ? 4 : strips * blocks >= 2 * n_cu || gated ? 2 : 1;
  const int wgs = (strips + f.ns - 1) / f.ns * blocks;
  f.S = n_cu / wgs;
  if (f.S > units / GW) f.S = units / GW;
  if (f.S < 1) f.S = 1;
  return f;
}
size_t sp_fp4_product_floats(int M, int N, int K, bool gated, int n_cu) {
  const Fp4Split f = split_of(M, N, K, gated, n_cu);
  return f.S > 1 ? (size_t)f.S * M * N : 0;
}

template <int MT, int NS, int OUT, bool XFRAG>
static void go(const Fp4GemmArgs& a, hipStream_t st) {
  const int sgs = (a.groups * a.S + 7) / 8 * 8;
  const dim3 grid(sgs * a.row_blocks), block(64 * GW);
  if (a.row_blocks == 1) hipLaunchKernelGGL((k_fp4_gemm<MT, NS, OUT, XFRAG, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_fp4_gemm<MT, NS, OUT, XFRAG, false>), grid, block, 0, st, a);
}
template <int OUT, bool XFRAG>
static hipError_t launch(const Fp4Split& f, Fp4GemmArgs& a, hipStream_t st) {
  const int per = OUT == OUT_GATED ? f.ns / 2 : f.ns, have = OUT == OUT_GATED ? a.N / 32 : a.N / 16;
  a.groups = (have + per - 1) / per;
  a.row_blocks = (a.M + 16 * f.mt - 1) / (16 * f.mt);
#define SP_FP4_MT(NSV)                                                                          \
  switch (f.mt) {                                                                               \
    case 1: go<1, NSV, OUT, XFRAG>(a, st); break;                                               \
    case 2: go<2, NSV, OUT, XFRAG>(a, st); break;                                               \
    default: go<4, NSV, OUT, XFRAG>(a, st); break;                                              \
  }
  if (f.ns == 4) SP_FP4_MT(4)
  else if (f.ns == 2) SP_FP4_MT(2)
  else if constexpr (OUT != OUT_GATED) SP_FP4_MT(1)
#undef SP_FP4_MT
  return hipGetLastError();
}

hipError_t sp_launch_fp4_parts(const bf16_t* X, bool frag, const void* W, float* out, int M, int N, int K, int n_cu, size_t part_floats,
                               int* S_out, hipStream_t st) {
  Fp4Split f = split_of(M, N, K, false, n_cu);
  while (f.S > 1 && (size_t)f.S * M * N > part_floats) --f.S;
  if ((size_t)f.S * M * N > part_floats) return hipErrorInvalidValue;
  *S_out = f.S;
  Fp4GemmArgs a{X, (const char*)W, out, M, N, K, (K + UNIT_K - 1) / UNIT_K, f.S, 0, 0, false};
  return frag ? launch<OUT_PARTS, true>(f, a, st) : launch<OUT_PARTS, false>(f, a, st);
}
hipError_t sp_launch_fp4_gateup(const bf16_t* X, bool frag, const void* W, bf16_t* act, int M, int F, int K, int n_cu, hipStream_t st) {
  Fp4Split f = split_of(M, 2 * F, K, true, n_cu);
  f.S = 1;
  Fp4GemmArgs a{X, (const char*)W, act, M, 2 * F, K, (K + UNIT_K - 1) / UNIT_K, 1, 0, 0, frag};
  return frag ? launch<OUT_GATED, true>(f, a, st) : launch<OUT_GATED, false>(f, a, st);
}
hipError_t sp_launch_fp4_product(const bf16_t* X, const void* W, bool gated, bf16_t* out, float* part, int M, int N, int K, int n_cu,
                                 hipStream_t st) {
  Fp4Split f = split_of(M, N, K, gated, n_cu);
  Fp4GemmArgs a{X, (const char*)W, out, M, N, K, (K + UNIT_K - 1) / UNIT_K, f.S, 0, 0, false};
  if (f.S == 1) return gated ? launch<OUT_GATED, false>(f, a, st) : launch<OUT_ROWS, false>(f, a, st);
  a.out = part;
  hipError_t e = launch<OUT_PARTS, false>(f, a, st);
  if (e != hipSuccess) return e;
  const size_t four = (size_t)M * (gated ? N / 2 : N) / 4;
  const dim3 grid((unsigned)((four + 255) / 256 < 4096 ? (four + 255) / 256 : 4096));
  if (gated) hipLaunchKernelGGL(k_fp4_fold<true>, grid, dim3(256), 0, st, part, out, f.S, M, N);
  else hipLaunchKernelGGL(k_fp4_fold<false>, grid, dim3(256), 0, st, part, out, f.S, M, N);
  return hipGetLastError();
}
