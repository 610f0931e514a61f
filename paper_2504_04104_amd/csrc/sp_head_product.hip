// Products head by head: out[m][h] = x[m][h] W[h]^T, bf16 with float32 sums.
#include "sp_launch.h"

// A wave has 16 rows x 16 columns of a head: a k step of 32 is one v_mfma_f32_16x16x32_bf16, both operands as they lie in memory.
// grid: (ceil(m / 16), ceil(n / 64), heads)
__global__ void __launch_bounds__(256) k_head_product(HeadProductArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, kg = lane >> 4;
  const int m0 = blockIdx.x * 16, n0 = blockIdx.y * 64 + wave * 16, h = blockIdx.z;
  if (n0 >= a.n) return;
  const bf16_t* x = a.x + (size_t)min(m0 + l15, a.m - 1) * a.x_row + h * a.x_head + kg * 8;
  const bf16_t* w = a.w + ((size_t)h * a.n + n0 + l15) * a.k + kg * 8;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.k; k += 32) {
    const u32x4_t xf = *reinterpret_cast<const u32x4_t*>(x + k), wf = *reinterpret_cast<const u32x4_t*>(w + k);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf), __builtin_bit_cast(bf16x8_t, xf), acc, 0, 0, 0);
  }
  // acc[i]: column n0 + kg * 4 + i of row m0 + l15
  if (m0 + l15 < a.m)
    *reinterpret_cast<uint2*>(a.out + (size_t)(m0 + l15) * a.out_row + h * a.out_head + n0 + kg * 4) = uint2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
}

hipError_t sp_launch_head_product(const HeadProductArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(k_head_product, dim3((a.m + 15) / 16, (a.n + 63) / 64, a.heads), dim3(256), 0, st, a);
  return hipGetLastError();
}
