// Products head by head: out[m][h] = x[m][h] W[h]^T, bf16 with float32 sums.
//
// Every weight is used m times and every value of x n times: up to some hundred rows the call is bound by the weights' and results' way
// through memory, and by its launch.  One row x 16 heads, 128 -> 512: 3.1 us; 64 rows x 64 heads, 512 -> 128: 7.6 (14 MB; half of the CUs have a
// workgroup, whose four steps wait for their loads one after the other); 637 x 64, 128 -> 512: 14.6 (61 MB, 4.2 TB/s, two thirds of it results);
// 2048 x 64 37 (176 MB, 4.7 TB/s).  These are kernels alone over three sets of inputs in turn; pairs below are of one set over and over, which
// is faster where the caches have it.
#include "sp_launch.h"

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

// ---- up to 16 rows: a wave has 16 rows x 16 columns of a head ------------------------------
// A k step of 32 is one v_mfma_f32_16x16x32_bf16, both operands as they lie in memory; eight steps' loads on their way at a time.
// grid: (heads, ceil(n / 64))
__global__ void __launch_bounds__(256) k_head_product_few(HeadProductArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, kg = lane >> 4;
  const int h = blockIdx.x, n0 = blockIdx.y * 64 + wave * 16;
  if (n0 >= a.n) return;
  const bf16_t* x = a.x + min(l15, a.m - 1) * a.x_row + h * a.x_head + kg * 8;
  const bf16_t* w = a.w + ((size_t)h * a.n + n0 + l15) * a.k + kg * 8;
  f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  int k = 0;
  auto steps = [&](auto& xf, auto& wf, int n) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
      xf[i] = *reinterpret_cast<const u32x4_t*>(x + k + i * 32);
      wf[i] = *reinterpret_cast<const u32x4_t*>(w + k + i * 32);
    }
#pragma unroll
    for (int i = 0; i < n; ++i)
      acc[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf[i]), __builtin_bit_cast(bf16x8_t, xf[i]), acc[i & 1], 0, 0, 0);
    k += n * 32;
  };
  u32x4_t xf[8], wf[8];
  while (k + 256 <= a.k) steps(xf, wf, 8);
  if (k + 128 <= a.k) steps(xf, wf, 4);
  while (k < a.k) steps(xf, wf, 1);
  const f32x4_t y = acc[0] + acc[1];
  // y[i]: column n0 + kg * 4 + i of row l15
  if (l15 < a.m)
    *reinterpret_cast<uint2*>(a.out + l15 * a.out_row + h * a.out_head + n0 + kg * 4) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

// ---- more: a workgroup has 64 rows x BN columns of a head -----------------------------------
// Steps of 128 columns of x and W by way of LDS, rows of 256 bytes whose 16-byte units are exchanged by the row's number; three
// workgroups a CU, so that one's loads pass behind another's products.  The result goes through LDS too, out as whole lines.
// grid: (heads, ceil(n / BN), ceil(m / 64)): the blocks of a head share an XCD's L2 (where heads are a multiple of eight)
__device__ __forceinline__ int swap256(int row) { return (row & 3) * 4 + ((row >> 2) & 3); }
template <int BN>
__global__ void __launch_bounds__(256) k_head_product(HeadProductArgs a) {
  constexpr int CT = BN / 64;                      // tiles of 32 columns a wave
  __shared__ __attribute__((aligned(16))) char s_w[BN * 256], s_x[64 * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l15 = lane & 15, kg = lane >> 4, l31 = lane & 31, hh = lane >> 5;
  const int h = blockIdx.x, n0 = blockIdx.y * BN, m0 = blockIdx.z * 64;
  const int rows = min(64, a.m - m0), cols = min(BN, a.n - n0);
  const auto wb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(a.w) + ((size_t)h * a.n + n0) * a.k, (short)0, cols * a.k * 2, 0x00020000);
  const int wr = wave & 1, wc = wave >> 1;         // the wave's 32 rows and its half of the columns
  f32x16_t acc[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
  const int fx = (wr * 32 + l31) * 256 + (hh ^ swap256(l31)) * 16, fw = (wc * CT * 32 + l31) * 256 + (hh ^ swap256(l31)) * 16;
  for (int k0 = 0; k0 < a.k; k0 += 128) {
    if (k0 > 0) __syncthreads();
    // a load is four rows; columns past the end, and rows, come as zeros
#pragma unroll
    for (int i = 0; i < BN / 16; ++i) {
      const int row = wave * (BN / 4) + i * 4 + kg, col = k0 + (l15 ^ swap256(row)) * 8;
      load_to_lds(wb, s_w + (wave * (BN / 4) + i * 4) * 256, col < a.k ? (row * a.k + col) * 2 : 0x7ffffff0, 0);
    }
    u32x4_t xr[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = wave * 16 + i * 4 + kg, col = k0 + (l15 ^ swap256(row)) * 8;
      xr[i] = (u32x4_t){0u, 0u, 0u, 0u};
      if (row < rows && col < a.k) xr[i] = *reinterpret_cast<const u32x4_t*>(a.x + (m0 + row) * a.x_row + h * a.x_head + col);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4_t*>(s_x + (wave * 16 + i * 4 + kg) * 256 + l15 * 16) = xr[i];
    SP_WAIT_VMEM(0);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(s_x + (fx ^ (s * 32)));
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(s_w + (fw ^ (s * 32)) + t * 8192);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc[t], 0, 0, 0);
      }
    }
  }
  __syncthreads();
  // acc[t][4 j ..]: columns (wc * CT + t) * 32 + j * 8 + hh * 4 .. of row wr * 32 + l31.  Rows of BN columns, units of 16 bytes exchanged.
  constexpr int UN = BN / 8;
  auto place = [](int row, int unit) { return row * BN * 2 + ((unit ^ row) & (UN - 1)) * 16; };
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint2*>(s_w + place(wr * 32 + l31, (wc * CT + t) * 4 + j) + hh * 8) =
          uint2{pack_bf16x2(acc[t][4 * j], acc[t][4 * j + 1]), pack_bf16x2(acc[t][4 * j + 2], acc[t][4 * j + 3])};
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64 * UN / 256; ++i) {
    const int p = i * 256 + threadIdx.x, row = p / UN, unit = p % UN;
    if (row < rows && unit * 8 < cols)
      *reinterpret_cast<u32x4_t*>(a.out + (m0 + row) * a.out_row + h * a.out_head + n0 + unit * 8) = *reinterpret_cast<const u32x4_t*>(s_w + place(row, unit));
  }
}

// ---- many rows, k 64, 128, 192 or 256: a wave keeps 64 columns of a head in registers ---------------------------
// Blocks of 32 rows come by one after the other by way of LDS, two places in turn, the next one's loads beside a block's products.  Four
// waves of a workgroup have neighbouring columns of the same rows.  The result goes out as whole lines by way of the wave's part of LDS.
// grid: (heads, ceil(n / 256), S): workgroup z has blocks z, z + S, ...
template <int K>
__global__ void __launch_bounds__(256) k_head_product_rows(HeadProductArgs a) {
  constexpr int S = K / 16, UN = K / 8, V = K / 64;    // steps, 16-byte units of a row, units of a block a thread
  __shared__ __attribute__((aligned(16))) char s_x[2][32 * K * 2], s_out[4][32 * 128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l31 = lane & 31, hh = lane >> 5;
  const int h = blockIdx.x, n0 = blockIdx.y * 256 + wave * 64, blocks = (a.m - 1) / 32 + 1;
  const bool idle = n0 >= a.n;                     // (a workgroup's last waves: they bring rows)
  u32x4_t xr[V];
  auto load = [&](int block) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int p = i * 256 + threadIdx.x, row = p / UN, unit = p % UN;
      xr[i] = *reinterpret_cast<const u32x4_t*>(a.x + min(block * 32 + row, a.m - 1) * a.x_row + h * a.x_head + unit * 8);
    }
  };
  auto place = [&](char* to) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int p = i * 256 + threadIdx.x, row = p / UN, unit = p % UN;
      *reinterpret_cast<u32x4_t*>(to + row * K * 2 + (unit ^ (row & 7)) * 16) = xr[i];
    }
  };
  load(blockIdx.z);
  u32x4_t wf[2][S];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < S; ++s) wf[t][s] = *reinterpret_cast<const u32x4_t*>(a.w + ((size_t)h * a.n + (idle ? 0 : n0) + t * 32 + l31) * K + s * 16 + hh * 8);
  char* mine = s_out[wave];
  place(s_x[0]);
  __syncthreads();
  for (int block = blockIdx.z, turn = 0; block < blocks; block += gridDim.z, turn ^= 1) {
    const bool more = block + (int)gridDim.z < blocks;
    if (more) load(block + gridDim.z);
    const char* x = s_x[turn] + l31 * K * 2;
    f32x16_t acc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const u32x4_t xf = *reinterpret_cast<const u32x4_t*>(x + ((s * 2 + hh) ^ (l31 & 7)) * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, wf[t][s]), __builtin_bit_cast(bf16x8_t, xf), acc[t], 0, 0, 0);
    }
    // acc[t][4 j ..]: columns t * 32 + j * 8 + hh * 4 .. of row l31
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint2*>(mine + l31 * 128 + ((t * 4 + j) ^ (l31 & 7)) * 16 + hh * 8) =
            uint2{pack_bf16x2(acc[t][4 * j], acc[t][4 * j + 1]), pack_bf16x2(acc[t][4 * j + 2], acc[t][4 * j + 3])};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + (lane >> 3), unit = lane & 7, at = block * 32 + row;
      const u32x4_t y = *reinterpret_cast<const u32x4_t*>(mine + row * 128 + (unit ^ (row & 7)) * 16);
      if (at < a.m && !idle) *reinterpret_cast<u32x4_t*>(a.out + at * a.out_row + h * a.out_head + n0 + unit * 8) = y;
    }
    if (more) place(s_x[turn ^ 1]);
    __syncthreads();
  }
}

// Two workgroups a CU (64 heads, 640 rows, 128 -> 512: 14.5 us, one a CU 15.3, three 15.1).  Taken where they have blocks enough to fill their
// registers for, by k (us, the kernel above and this one): 64 -> 512, 64 heads, 33 rows 3.8 and
// 3.4, 640 rows 18.2 and 11.2; 128 -> 512 128 rows 5.7 and 7.0, 256 rows 9.6 and 9.3, 640 rows 18.0 and 14.5, 128 heads 46.8 and 23.5; 192 -> 512
// 128 rows 7.6 and 9.0, 256 rows 13.7 and 11.5; 256 -> 256 640 rows 14.7 and 15.6, 2048 rows 37.0 and 28.0.
inline bool rows_fill(const HeadProductArgs& a, long long least) {
  return a.n % 64 == 0 && ((a.m - 1) / 32 + 1) * (long long)a.heads * ((a.n + 255) / 256) >= least;
}
template <int K>
static hipError_t go_rows(const HeadProductArgs& a, hipStream_t st) {
  const int blocks = (a.m - 1) / 32 + 1, one = a.heads * ((a.n + 255) / 256);
  int s = (512 + one - 1) / one;
  if (s > blocks) s = blocks;
  hipLaunchKernelGGL(k_head_product_rows<K>, dim3(a.heads, (a.n + 255) / 256, s), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t sp_launch_head_product(const HeadProductArgs& a, hipStream_t st) {
  // Few rows, and a workgroup a CU at most (16 rows: 16 heads 128 -> 512 3.0 us, in blocks of 64 rows 3.3; 128 heads 5.9 and 4.3).
  if (a.m <= 16 && (long long)a.heads * ((a.n + 63) / 64) <= 256) {
    hipLaunchKernelGGL(k_head_product_few, dim3(a.heads, (a.n + 63) / 64), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  if (a.k == 64 && a.m > 16 && rows_fill(a, 256)) return go_rows<64>(a, st);
  if (a.k == 128 && rows_fill(a, 1024)) return go_rows<128>(a, st);
  if (a.k == 192 && rows_fill(a, 1024)) return go_rows<192>(a, st);
  if (a.k == 256 && rows_fill(a, 2048)) return go_rows<256>(a, st);
  // (blocks of rows in several launches where there are more than a grid takes)
  for (long long m0 = 0; m0 < a.m; m0 += 64 * 65535) {
    HeadProductArgs b = a;
    b.x += m0 * a.x_row;
    b.out += m0 * a.out_row;
    b.m = (int)(a.m - m0 < 64 * 65535 ? a.m - m0 : 64 * 65535);
    const int blocks = (b.m + 63) / 64;
    // 128 columns where that leaves two workgroups a CU (64 heads 512 -> 128: 640 rows 14.3 us, 64 columns 16.9; 256 rows 8.5 and 7.8)
    if (a.n > 64 && (long long)a.heads * blocks * ((a.n + 127) / 128) >= 512)
      hipLaunchKernelGGL(k_head_product<128>, dim3(a.heads, (a.n + 127) / 128, blocks), dim3(256), 0, st, b);
    else
      hipLaunchKernelGGL(k_head_product<64>, dim3(a.heads, (a.n + 63) / 64, blocks), dim3(256), 0, st, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
