// Products of bf16 rows with a matrix of 4-bit weights (sp_fp4.h): out[m][n] = sum_k X[m][k] W[n][k], W as the values that its
// codes and scales stand for, sums in float32.
//
// Weights lie in units of 16 rows x 256 columns, 2176 bytes in a row of memory: twice 64 x 16 bytes of codes, lane l of a wave
// taking row l % 16 and the 32 columns (l / 16) * 32 .. of either half -- one group, one scale -- and 64 x 2 bytes of scales.
// The units of 16 rows (a strip) follow each other over the columns.  Which column of X a product's operand holds is free as long
// as both sides agree: the four steps over a half take columns kg * 32 + j * 8 .. + 7 in lane kg.  A conversion instruction makes
// two codes and their scale two bf16 values.
//
// Two kernels: up to 16 rows of short products the waves of a workgroup share strips and cut the columns among them; elsewhere
// they have strips of their own and share rows of X through LDS.  What bounds them: up to some forty rows the weights' way from
// memory (one row of 28672 x 4096, 62 MB, 14.6 us; of 57344 x 8192, 249 MB, 45.9 us, 5.4 TB/s); more rows, the rows' way through
// L2 and LDS into the matrix cores (64 rows of 28672 x 4096 20.4 us; 200 rows of 57344 x 8192 170 us, 1.1 PFLOP/s).
#include "sp_launch.h"
#include "sp_fp4.h"
#include "sp_fp4_split.h"

enum { OUT_PARTS, OUT_ROWS, OUT_GATED };

struct Fp4GemmArgs {
  const bf16_t* X;
  const char* W;
  void* out;                 // OUT_PARTS: float32 [S][M][N]; OUT_ROWS: bf16 [M][N]; OUT_GATED: bf16 [M][N / 2]
  int M, N, K, units, S;
  int tiles, row_blocks;     // workgroups over the strips; over the rows
  bool frag, frag_out;       // X in fragment order, rows of units * UNIT_K columns, or row-major; OUT_GATED: the result's order
};

__device__ __forceinline__ float silu(float x) { return x / (1.f + __expf(-x)); }

// Up to 16 rows: the waves of a workgroup share NS strips and cut the columns among them; their sums are added through LDS.
// Rows and weights come from memory in fragment order or as they are, PF units ahead: loads return in order, so that rows that are
// asked for later than weights wait for those.
// OUT_GATED: a strip is eight gate rows and the eight up rows that belong to them, lanes 0-7 and 8-15 of sixteen.
template <int NS, int OUT, bool XFRAG>
__global__ void __launch_bounds__(NS <= 2 ? 512 : 256) k_fp4_few(Fp4GemmArgs a) {
  constexpr int NW = NS <= 2 ? 8 : 4, PF = NS <= 2 ? 4 : 2;
  __shared__ f32x4_t s_sum[NW][NS][64];
  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63, l15 = lane & 15, kg = lane >> 4;
  const int slice = uni((int)blockIdx.x / a.tiles), strip0 = uni(((int)blockIdx.x - slice * a.tiles) * NS);
  const int strips = a.N >> 4;
  const int su0 = slice * a.units / a.S, su1 = (slice + 1) * a.units / a.S;
  const int u0 = uni(su0 + (su1 - su0) * wave / NW), u1 = uni(su0 + (su1 - su0) * (wave + 1) / NW);

  // Buffers: loads past the run, past the strips and past the rows return zeros without a memory access.  What is to be checked
  // is in the lane's offset: a scalar one is not part of the check.
  const int xk = XFRAG ? a.units * UNIT_K : a.K;
  const auto xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(a.X), (short)0, (XFRAG ? 16 : a.M) * xk * 2, 0x00020000);
  const int x_lane = XFRAG ? kg * 1024 + l15 * 16 : l15 * xk * 2 + kg * 64;
  const int half = OUT == OUT_GATED ? (strips >> 1) * a.units * UNIT_BYTES : 0;              // from the gate rows to the up rows
  u32x4_t xf[PF][8], wq[PF][NS][2];
  uint32_t wsc[PF][NS];
  auto fetch = [&](int p, int u) {
    const bool run = u < u1;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int strip = strip0 + i;
      const bool on = run && strip < strips;
      const int unit_strip = OUT == OUT_GATED ? strip >> 1 : strip;
      const auto wb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.W) + ((size_t)(on ? unit_strip : 0) * a.units + (on ? u : 0)) * UNIT_BYTES,
                                                        (short)0, on ? half + UNIT_BYTES : 0, 0x00020000);
      int at = lane, up = 0;
      if (OUT == OUT_GATED) { at = kg * 16 + (strip & 1) * 8 + (l15 & 7); up = l15 < 8 ? 0 : half; }
#pragma unroll
      for (int b = 0; b < 2; ++b) wq[p][i][b] = __builtin_amdgcn_raw_buffer_load_b128(wb, up + at * 16 + b * 1024, 0, 2);
      wsc[p][i] = __builtin_amdgcn_raw_buffer_load_b16(wb, up + at * 2 + 2048, 0, 2);
    }
#pragma unroll
    for (int step = 0; step < 8; ++step) {
      const int k0 = (run ? u : 0) * UNIT_K + (step >> 2) * 128;
      const int at = XFRAG ? (k0 >> 5) * 1024 + (step & 3) * 256 : k0 * 2 + (step & 3) * 16;
      // (row-major: columns past the end meet weights of zero, but what lies behind a row may be anything)
      const int off = run && (XFRAG || k0 + kg * 32 < a.K) ? x_lane : 0x7fffff00;
      xf[p][step] = __builtin_amdgcn_raw_buffer_load_b128(xb, off, at, 0);
    }
  };
#pragma unroll
  for (int p = 0; p < PF; ++p) fetch(p, u0 + p);
  f32x4_t acc[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) acc[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  for (int ub = u0; ub < u1; ub += PF) {
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      if (ub + p < u1) {
#pragma unroll
        for (int step = 0; step < 8; ++step) {
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            const u32x4_t wf = fp4_to_bf16x8(wq[p][i][step >> 2][step & 3], fp4_scale((wsc[p][i] >> (8 * (step >> 2))) & 255u));
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf), __builtin_bit_cast(bf16x8_t, xf[p][step]),
                                                             acc[i], 0, 0, 0);
          }
        }
        fetch(p, ub + p + PF);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NS; ++i) s_sum[wave][i][lane] = acc[i];
  __syncthreads();
  // a lane's four sums: row l15 of X, rows kg * 4 .. + 3 of the strip
  auto total = [&](int i, int ln) {
    f32x4_t v = s_sum[0][i][ln];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += s_sum[w][i][ln];
    return v;
  };
  const int strip = strip0 + wave;
  if (wave >= NS || strip >= strips || l15 >= a.M || (OUT == OUT_GATED && lane >= 32)) return;
  const f32x4_t v = total(wave, lane);
  if constexpr (OUT == OUT_GATED) {
    const f32x4_t up = total(wave, lane + 32);
    *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + row_at(a.frag_out, l15, strip * 8 + kg * 4, a.N >> 1)) =
        uint2{pack_bf16x2(silu(v[0]) * up[0], silu(v[1]) * up[1]), pack_bf16x2(silu(v[2]) * up[2], silu(v[3]) * up[3])};
  } else if constexpr (OUT == OUT_PARTS) {
    *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + ((size_t)slice * a.M + l15) * a.N + strip * 16 + kg * 4) = v;
  } else {
    *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + (size_t)l15 * a.N + strip * 16 + kg * 4) =
        uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
}

// The waves share the rows of X through LDS, which a load brings there without registers, and have NS strips each over all columns
// of the slice.  A chunk is 128 columns, half a unit; loads are three chunks ahead (five are no faster), a chunk's rows before its
// weights, and go out between the products: all at once behind the barrier they held up the matrix cores (4096 x 14336, 64 rows,
// four tiles and four strips whole 91.8 us, 83.3 between).  Up to two tiles, two groups of four waves take a chunk in turn and add
// their sums through LDS: two waves a SIMD, half the steps (64 rows of 4096 x 4096 10.4 -> 8.6 us); with more tiles that is level.
#define PANELS 4
#define AHEAD 3
constexpr int groups_of(int mt) { return mt <= 2 ? 2 : 1; }
template <int MT, int NS, int OUT>
__global__ void __launch_bounds__(256 * groups_of(MT), MT * NS <= 16 ? 2 : 1) k_fp4_many(Fp4GemmArgs a) {
  constexpr int G = groups_of(MT), PANEL = MT * 4096, LOADS = MT + 2 * NS;
  // arrays of their own, so that the compiler knows which loads a read has to wait for
  __shared__ __attribute__((aligned(16))) char p0[G * PANEL];
  __shared__ __attribute__((aligned(16))) char p1[G * PANEL];
  __shared__ __attribute__((aligned(16))) char p2[G * PANEL];
  __shared__ __attribute__((aligned(16))) char p3[G * PANEL];
#define SP_PAN(i) (((i) == 0 ? p0 : (i) == 1 ? p1 : (i) == 2 ? p2 : p3) + grp * PANEL)
  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int grp = G == 1 ? 0 : uni((int)threadIdx.x >> 8), wave = uni((int)threadIdx.x >> 6) & 3, lane = threadIdx.x & 63, l15 = lane & 15, kg = lane >> 4;
  // the row blocks of a column tile on one XCD, one after the other
  const int id = blockIdx.x, local = id >> 3;
  const int rb = uni(local % a.row_blocks), ts = uni((local / a.row_blocks) * 8 + (id & 7));
  const int slice = uni(ts / a.tiles), tile = uni(ts - slice * a.tiles);
  if (slice >= a.S) return;
  const int c_begin = uni((int)((long long)slice * a.units / a.S) * 2), c_end = uni(min((int)((long long)(slice + 1) * a.units / a.S) * 2, (a.K + 127) / 128));
  const int strips = a.N >> 4, t0 = rb * MT;
  // gated: the first half of the wave's strips are gate rows, the second the up rows of the same columns
  const int own = OUT == OUT_GATED ? NS / 2 : NS, strip0 = (tile * 4 + wave) * own;
  const int strip_bytes = a.units * UNIT_BYTES;
  const char* w[NS];
  int live[NS];              // bytes
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int strip = strip0 + i % own + i / own * (strips >> 1);
    live[i] = strip0 + i % own < (OUT == OUT_GATED ? strips >> 1 : strips) ? strip_bytes : 0;
    w[i] = a.W + (live[i] ? (size_t)strip * strip_bytes : 0);
  }
  // A load to LDS brings eight rows x 64 columns of a tile, the wave's of its four: lane l 16 bytes (a piece) of row l / 8.  They
  // are whole lines of X, row-major or in fragment order (64 rows of 28672 x 4096 21.7 us, by 32 columns of 16 rows 23.3).  The
  // pieces of a row are exchanged by the row's number, for reads without bank conflicts.  Rows past the last, and columns (of the
  // last chunk) past the end, are past the buffer's end: zeros.
  const int r8 = lane >> 3, piece = (lane & 7) ^ r8 ^ (wave & 1), x_row = (wave & 1) * 8 + r8, x_col = (wave >> 1) * 64 + piece * 8;
  const int xk = a.frag ? a.units * UNIT_K : a.K, x_step = a.frag ? 4096 : 256;
  const int x_rows = min(a.M - t0 * 16, MT * 16), x_bytes = (a.frag ? (x_rows + 15) & ~15 : x_rows) * xk * 2;
  const bf16_t* xblk = a.X + (size_t)t0 * 16 * xk;
  const int x_lane = a.frag ? (x_col >> 5) * 1024 + (piece & 3) * 256 + x_row * 16 : (x_row * xk + x_col) * 2;
  const int c_part = a.K % 128 ? a.K / 128 : -1, x_part = x_col < a.K % 128 ? x_lane : 0x7fffff00;
  const int lane16 = lane * 16;
  int read_at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) read_at[j] = ((kg >> 1) * 2 + (l15 >> 3)) * 1024 + (l15 & 7) * 128 + (((kg & 1) * 4 + j) ^ (l15 & 7) ^ (l15 >> 3)) * 16;
  // the groups take a chunk in turn: chunk of step i, and half of the unit it is
#define SP_C(i) (c_begin + G * (i) + grp)
#define SP_HALF(I) (G == 1 ? (I) & 1 : grp)
  const int steps = (c_end - c_begin + G - 1) / G;
  // the word with the lane's two scales, and the turn that brings the first into the exponent field
  const int scale_at = 2048 + (lane & 62) * 2, turn = (lane & 1) * 16 + 9;
  u32x4_t wb[PANELS][NS];
  uint32_t ws[PANELS][NS];
  f32x4_t acc[MT][NS];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NS; ++i) acc[t][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#define SP_LOAD_X(I, C)                                                                                                \
  {                                                                                                                    \
    const auto xb_ = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(xblk), (short)0, (C) < c_end ? x_bytes : 0, 0x00020000); \
    const int x_ = (C) == c_part ? x_part : x_lane;                                                                    \
    _Pragma("unroll") for (int t = 0; t < MT; ++t)                                                                     \
        load_to_lds(xb_, SP_PAN(I) + (t * 4 + wave) * 1024, x_ + t * 32 * xk, (C) * x_step);                           \
  }
#define SP_LOAD_W(I, C, s)                                                                                             \
  {                                                                                                                    \
    const auto wr_ = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(w[s]), (short)0, (C) < c_end ? live[s] : 0, 0x00020000); \
    wb[I][s] = __builtin_amdgcn_raw_buffer_load_b128(wr_, lane16 + SP_HALF(I) * 1024, ((C) >> 1) * UNIT_BYTES, 0);      \
    ws[I][s] = __builtin_amdgcn_raw_buffer_load_b32(wr_, scale_at, ((C) >> 1) * UNIT_BYTES, 0);                        \
  }
#define SP_READ(I, j, Q)                                                                                               \
  _Pragma("unroll") for (int t = 0; t < MT; ++t)                                                                       \
      xq[Q][t] = *reinterpret_cast<const u32x4_t*>(SP_PAN(I) + t * 4096 + read_at[j]);
  // A quarter of a chunk's products, between them the reads for the next quarter and a part of the loads
#define SP_STEP(I, j, LOADS)                                                                                           \
  {                                                                                                                    \
    if ((j) < 3) { SP_READ(I, (j) + 1, ((j) + 1) & 1) } else { SP_READ(((I) + 1) % PANELS, 0, 0) }                     \
    LOADS                                                                                                              \
    _Pragma("unroll") for (int i = 0; i < NS; ++i) {                                                                   \
      const u32x4_t wf = fp4_to_bf16x8(wb[I][i][j], __uint_as_float(__builtin_amdgcn_alignbit(ws[I][i], ws[I][i], turn + SP_HALF(I) * 8))); \
      _Pragma("unroll") for (int t = 0; t < MT; ++t)                                                                   \
          acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf),                        \
                                                              __builtin_bit_cast(bf16x8_t, xq[(j) & 1][t]), acc[t][i], 0, 0, 0); \
    }                                                                                                                  \
    __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);                                                                 \
    _Pragma("unroll") for (int n = 0; n < MT * NS; ++n) {                                                              \
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                                               \
      __builtin_amdgcn_sched_group_barrier(0x002, MT <= 4 ? 2 : 1, 0);                                                 \
      if (n % NS == 0) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                              \
      if (n % NS == 1) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                              \
    }                                                                                                                  \
    __builtin_amdgcn_sched_barrier(0);                                                                                 \
  }
#define SP_CHUNK(I, C)                                                                                                 \
  {                                                                                                                    \
    SP_WAIT_VMEM((AHEAD - 2) * LOADS + 2 * NS);                                                                        \
    bare_barrier();                                                                                                    \
    const int ahead_ = SP_C((C) + AHEAD);                                                                              \
    SP_STEP(I, 0, SP_LOAD_X(((I) + AHEAD) % PANELS, ahead_))                                                           \
    SP_STEP(I, 1, _Pragma("unroll") for (int s = 0; s < NS; s += 2) SP_LOAD_W(((I) + AHEAD) % PANELS, ahead_, s)) \
    SP_STEP(I, 2, _Pragma("unroll") for (int s = 1; s < NS; s += 2) SP_LOAD_W(((I) + AHEAD) % PANELS, ahead_, s)) \
    SP_STEP(I, 3, )                                                                                                    \
  }
#define SP_CHUNK_PRODUCTS(I) { SP_STEP(I, 0, ) SP_STEP(I, 1, ) SP_STEP(I, 2, ) SP_STEP(I, 3, ) }
#pragma unroll
  for (int p = 0; p < AHEAD; ++p) {
    SP_LOAD_X(p, SP_C(p))
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < NS; ++s) SP_LOAD_W(p, SP_C(p), s)
    __builtin_amdgcn_sched_barrier(0);
  }
  SP_WAIT_VMEM((AHEAD - 1) * LOADS + 2 * NS);
  bare_barrier();
  u32x4_t xq[2][MT];
  SP_READ(0, 0, 0)
  int c = 0;
  for (; c + PANELS <= steps; c += PANELS) {
    SP_CHUNK(0, c)
    SP_CHUNK(1, c + 1)
    SP_CHUNK(2, c + 2)
    SP_CHUNK(3, c + 3)
  }
  SP_WAIT_VMEM(0);
  if (c < steps) {                                  // up to three are left, and have been asked for
    bare_barrier();
    SP_CHUNK_PRODUCTS(0)
    if (c + 1 < steps) SP_CHUNK_PRODUCTS(1)
    if (c + 2 < steps) SP_CHUNK_PRODUCTS(2)
  }
#undef SP_CHUNK_PRODUCTS
#undef SP_STEP
#undef SP_LOAD_X
#undef SP_LOAD_W
#undef SP_CHUNK
#undef SP_READ
#undef SP_PAN
#undef SP_C
#undef SP_HALF
  if constexpr (G > 1) {
    // the second group's sums to the first, in the first panel's place
    static_assert(MT * NS * 4096 <= G * PANEL, "the sums of four waves");
    f32x4_t* const sums = reinterpret_cast<f32x4_t*>(p0) + wave * MT * NS * 64 + lane;
    __syncthreads();
    if (grp) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < NS; ++i) sums[(t * NS + i) * 64] = acc[t][i];
    }
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < NS; ++i) acc[t][i] += sums[(t * NS + i) * 64];
  }

  // a lane's four sums: row t * 16 + l15 of X, rows kg * 4 .. + 3 of the strip
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = (t0 + t) * 16 + l15;
    if (m >= a.M) continue;
#pragma unroll
    for (int i = 0; i < own; ++i) {
      if (!live[i]) continue;
      const f32x4_t v = acc[t][i];
      const int col = (strip0 + i) * 16 + kg * 4;
      if constexpr (OUT == OUT_GATED) {
        const f32x4_t up = acc[t][i + NS / 2];
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + row_at(a.frag_out, m, col, a.N >> 1)) =
            uint2{pack_bf16x2(silu(v[0]) * up[0], silu(v[1]) * up[1]), pack_bf16x2(silu(v[2]) * up[2], silu(v[3]) * up[3])};
      } else if constexpr (OUT == OUT_PARTS) {
        *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + ((size_t)slice * a.M + m) * a.N + col) = v;
      } else {
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + (size_t)m * a.N + col) =
            uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      }
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
size_t sp_fp4_bytes(int N, int K) { return fp4_bytes(N, K); }
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

size_t sp_fp4_product_floats(int M, int N, int K, int n_cu) {
  const Fp4Split f = fp4_split_call(M, N, K, n_cu);
  return f.S > 1 ? (size_t)f.S * M * N : 0;
}

template <int NS, int OUT>
static void go_few(Fp4GemmArgs& a, hipStream_t st) {
  a.tiles = (a.N / 16 + NS - 1) / NS;
  const dim3 grid(a.tiles * a.S), block(NS <= 2 ? 512 : 256);
  if constexpr (OUT == OUT_GATED)                   // (else row-major: rows of a call of its own, or one or two of a forward call)
    if (a.frag) { hipLaunchKernelGGL((k_fp4_few<NS, OUT, true>), grid, block, 0, st, a); return; }
  hipLaunchKernelGGL((k_fp4_few<NS, OUT, false>), grid, block, 0, st, a);
}
template <int MT, int NS, int OUT>
static void go_many(Fp4GemmArgs& a, hipStream_t st) {
  const int strips = OUT == OUT_GATED ? a.N / 32 : a.N / 16, per = OUT == OUT_GATED ? 2 * NS : 4 * NS;
  a.row_blocks = (a.M + 16 * MT - 1) / (16 * MT);
  a.tiles = (strips + per - 1) / per;
  hipLaunchKernelGGL((k_fp4_many<MT, NS, OUT>), dim3((a.tiles * a.S + 7) / 8 * 8 * a.row_blocks), dim3(256 * groups_of(MT)), 0, st, a);
}
template <int OUT>
static hipError_t launch(const Fp4Split& f, Fp4GemmArgs& a, hipStream_t st) {
  switch (f.mt * 8 + f.ns) {
    case 1: if constexpr (OUT != OUT_PARTS) { go_few<1, OUT>(a, st); break; } else return hipErrorInvalidValue;
    case 2: if constexpr (OUT != OUT_PARTS) { go_few<2, OUT>(a, st); break; } else return hipErrorInvalidValue;
    case 4: if (OUT != OUT_GATED && a.frag) return hipErrorInvalidValue; go_few<4, OUT>(a, st); break;
    case 1 * 8 + 2: go_many<1, 2, OUT>(a, st); break;
    case 2 * 8 + 2: go_many<2, 2, OUT>(a, st); break;
    case 4 * 8 + 2: go_many<4, 2, OUT>(a, st); break;
    case 4 * 8 + 4: go_many<4, 4, OUT>(a, st); break;
    case 5 * 8 + 4: go_many<5, 4, OUT>(a, st); break;
    case 7 * 8 + 4: go_many<7, 4, OUT>(a, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t sp_launch_fp4_parts(const bf16_t* X, bool frag, const void* W, float* out, int M, int N, int K, int n_cu, size_t part_floats,
                               int* S_out, hipStream_t st) {
  const Fp4Split f = fp4_split_parts(M, N, K, n_cu, part_floats);
  if (f.S < 1) return hipErrorInvalidValue;
  *S_out = f.S;
  Fp4GemmArgs a{X, (const char*)W, out, M, N, K, (K + UNIT_K - 1) / UNIT_K, f.S, 0, 0, frag, false};
  return launch<OUT_PARTS>(f, a, st);
}
hipError_t sp_launch_fp4_gateup(const bf16_t* X, bool frag, const void* W, bf16_t* act, int M, int F, int K, int n_cu, hipStream_t st) {
  const Fp4Split f = fp4_split_gateup(M, F, K, n_cu);
  Fp4GemmArgs a{X, (const char*)W, act, M, 2 * F, K, (K + UNIT_K - 1) / UNIT_K, 1, 0, 0, frag, frag};
  return launch<OUT_GATED>(f, a, st);
}
hipError_t sp_launch_fp4_product(const bf16_t* X, const void* W, bool gated, bf16_t* out, float* work, int M, int N, int K, int n_cu,
                                 hipStream_t st) {
  const Fp4Split f = fp4_split_call(M, N, K, n_cu);
  Fp4GemmArgs a{X, (const char*)W, out, M, N, K, (K + UNIT_K - 1) / UNIT_K, f.S, 0, 0, false, false};
  if (f.S == 1) return gated ? launch<OUT_GATED>(f, a, st) : launch<OUT_ROWS>(f, a, st);
  a.out = work;
  const hipError_t e = launch<OUT_PARTS>(f, a, st);
  if (e != hipSuccess) return e;
  const size_t four = (size_t)M * (gated ? N / 2 : N) / 4;
  const dim3 grid((unsigned)((four + 255) / 256 < 4096 ? (four + 255) / 256 : 4096));
  if (gated) hipLaunchKernelGGL(k_fp4_fold<true>, grid, dim3(256), 0, st, work, out, f.S, M, N);
  else hipLaunchKernelGGL(k_fp4_fold<false>, grid, dim3(256), 0, st, work, out, f.S, M, N);
  return hipGetLastError();
}
