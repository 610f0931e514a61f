// Rotary positions of rows of heads: (a, b) -> gain * (a cos - b sin, b cos + a sin) for the pairs of a head's first `dims` columns at
// the angle position * freq[pair]; the other columns are copied.  Back (sign -1): the transpose, the angle negated, which is also
// the gradient.
#include "sp_launch.h"

template <typename T, int V> struct Vec;
template <> struct Vec<float, 4> {
  static __device__ __forceinline__ void ld(const float* p, float (&v)[4]) {
    const f32x4_t u = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = u[i];
  }
  static __device__ __forceinline__ void st(float* p, const float (&v)[4]) { *reinterpret_cast<f32x4_t*>(p) = (f32x4_t){v[0], v[1], v[2], v[3]}; }
};
template <> struct Vec<bf16_t, 4> {
  static __device__ __forceinline__ void ld(const bf16_t* p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
  }
  static __device__ __forceinline__ void st(bf16_t* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
};
template <> struct Vec<bf16_t, 8> {
  static __device__ __forceinline__ void ld(const bf16_t* p, float (&v)[8]) {
    const u32x4_t u = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(u[i]); v[2 * i + 1] = bf16_hi(u[i]); }
  }
  static __device__ __forceinline__ void st(bf16_t* p, const float (&v)[8]) {
    *reinterpret_cast<u32x4_t*>(p) = (u32x4_t){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};

// A workgroup takes a.rows_per rows: the cosines and sines of all their pairs first (the angle in double precision, whole turns
// taken off there), then V columns a thread at a time together with V that they are paired with, or with V others that pass.  A stream in
// and out: 32749 rows of 8 heads of 128, bf16, 134 MB, 22.7 us, 5.9 TB/s (a large copy 5.1), float32, 16384 rows, 21.8; one row 2.5 and 2.7
// (kernels alone, three sets of inputs in turn; pairs below of one set over and over).
// As many rows as have a piece for every thread: 64 heads 1 row at a time 64 rows 4.0 us, 8192 41.0, 8 at a time 14.8 and 45.8; 8 heads 4 at a
// time 64 rows 3.2, 8192 7.2, 32749 21.6, 1 at a time 3.1, 9.7 and 28.4.
#define ROTATE_ROWS 8                              // at most
#define ROTATE_LAUNCH (1 << 23)                    // rows of a launch
template <typename T, int V>
__global__ void __launch_bounds__(256) k_rotate(RotateArgs a) {
  __shared__ float s_cos[ROTATE_ROWS][2 * SP_ROPE_PAIRS], s_sin[ROTATE_ROWS][2 * SP_ROPE_PAIRS];
  const long long row0 = (long long)blockIdx.x * a.rows_per;
  const int n_rows = (int)min((long long)a.rows_per, a.n_rows - row0), pairs = a.dims >> 1, half = a.d_head >> 1;
  for (int i = threadIdx.x; i < n_rows * pairs; i += 256) {
    const int r = i / pairs, t = i - r * pairs;
    const double turns = (double)a.pos[row0 + r] * a.freq[t] * 0.15915494309189535;
    const float ang = (float)((turns - rint(turns)) * 6.283185307179586);
    s_cos[r][t] = cosf(ang) * a.gain;
    s_sin[r][t] = sinf(ang) * a.gain * a.sign;
  }
  __syncthreads();
  const int units = half / V, per_row = a.n_heads * units;
  for (int i = threadIdx.x; i < n_rows * per_row; i += 256) {
    const int r = i / per_row, j = i - r * per_row, head = j / units, t = (j - head * units) * V;
    const bool halves = a.layout == 0, passes = halves && t >= pairs;
    const int ca = passes ? a.dims + t - pairs : t, cb = !halves ? half + t : passes ? a.dims + half - pairs + t - pairs : pairs + t;
    const T* x = reinterpret_cast<const T*>(a.x) + (row0 + r) * a.x_row + head * a.x_head;
    T* out = reinterpret_cast<T*>(a.out) + (row0 + r) * a.out_row + head * a.out_head;
    float u[V], v[V];
    Vec<T, V>::ld(x + ca, u);
    Vec<T, V>::ld(x + cb, v);
    if (halves && !passes) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float co = s_cos[r][t + e], si = s_sin[r][t + e], p = u[e], q = v[e];
        u[e] = p * co - q * si;
        v[e] = q * co + p * si;
      }
    } else if (!halves) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        if (ca + e < a.dims) {
          const float co = s_cos[r][(ca + e) / 2], si = s_sin[r][(ca + e) / 2], p = u[e], q = u[e + 1];
          u[e] = p * co - q * si;
          u[e + 1] = q * co + p * si;
        }
        if (cb + e < a.dims) {
          const float co = s_cos[r][(cb + e) / 2], si = s_sin[r][(cb + e) / 2], p = v[e], q = v[e + 1];
          v[e] = p * co - q * si;
          v[e + 1] = q * co + p * si;
        }
      }
    }
    Vec<T, V>::st(out + ca, u);
    Vec<T, V>::st(out + cb, v);
  }
}

hipError_t sp_launch_rotate(int dtype, RotateArgs& a, hipStream_t st) {
  const size_t elt = dtype == 0 ? 4 : 2;
  // sixteen-byte pieces of bf16 rows where neither the pairs nor the columns that pass end inside one
  const bool wide = a.d_head % 16 == 0 && (a.layout == 1 || a.dims % 16 == 0);
  const long long pieces = (long long)a.n_heads * (a.d_head / 2) / (dtype != 0 && wide ? 8 : 4);       // (of a row)
  a.rows_per = pieces >= 256 ? 1 : (int)(256 / pieces);
  if (a.rows_per > ROTATE_ROWS) a.rows_per = ROTATE_ROWS;
  // (in several launches where there are more rows than a grid takes)
  for (int rest = a.n_rows; rest > 0;) {
    a.n_rows = rest < ROTATE_LAUNCH ? rest : ROTATE_LAUNCH;
    const dim3 grid((a.n_rows + a.rows_per - 1) / a.rows_per), block(256);
    if (dtype == 0) hipLaunchKernelGGL((k_rotate<float, 4>), grid, block, 0, st, a);
    else if (wide) hipLaunchKernelGGL((k_rotate<bf16_t, 8>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_rotate<bf16_t, 4>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    rest -= a.n_rows;
    a.x = static_cast<const char*>(a.x) + (size_t)a.n_rows * a.x_row * elt;
    a.out = static_cast<char*>(a.out) + (size_t)a.n_rows * a.out_row * elt;
    a.pos += a.n_rows;
  }
  return hipSuccess;
}
