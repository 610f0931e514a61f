// How a product with 4-bit weights is stored and cut, made on the host.  Plain C++.
#pragma once
#include <stddef.h>

#define UNIT_K 256        // storage goes in units of 16 rows x 256 columns
#define UNIT_BYTES 2176

inline size_t fp4_bytes(int N, int K) { return (size_t)(N / 16) * ((K + UNIT_K - 1) / UNIT_K) * UNIT_BYTES; }

// Tiles of rows (0: the kernel for few rows) and strips of a workgroup, and slices of the columns, whose sums are joined by a launch
// of their own (`join` us; 0 where whoever takes the partial sums adds them up).  What is least by these times: a chunk of 128
// columns 0.22 us for one tile and two strips, 0.27 for two tiles, 0.40 and 0.66 for four with two and four strips, 0.82 for five,
// 1.12 for seven (over 14336 columns, 112 chunks, with at most one workgroup on a CU); a unit of a wave of the kernel for few
// rows 1 us and more with every row, and 0.8 more before them; a megabyte of partial sums 0.3.  Workgroups past the CUs take
// turns: two at a time on a CU are not faster than one after the other.  Us a call, as chosen and next to it (tiles x strips):
// 28672 x 4096 gated, 64 rows 4 x 2 20.4 (2 x 2 23.9, 4 x 4 27.4), 100 rows 4 x 4 28.4 (4 x 2 30.9), 160 rows 5 x 4 35.2 (4 x 4
// 45.2), 200 rows 7 x 4 45.4 (4 x 4 47.9), 256 rows 4 x 4 49.9 (7 x 4 84.2); 4096 x 14336, 17 rows 2 x 2 in 8 slices 13.2 (in 4
// 15.2, whole 35.8), 64 rows in 4 16.2 (in 8 18.0), 200 rows 4 x 4 in 4 31.9 (2 x 2 whole 37.5); 4096 x 4096, one row with the kernel
// for few rows 7.4 (one tile 8.3, in 4 slices 11.6), 64 rows one tile 8.6 (two 10.2, in 4 slices 11.6), 200 rows two tiles 11.0 (one
// 13.3); 4096 x 14336, one row with the kernel for few rows 11.6 (one tile in 8 slices 12.4), nine rows with one tile 12.7 (few rows'
// 14.8); 28672 x 4096 gated, one row with one tile 14.6 (few rows' 15.9), 16 rows 14.7 (19.9).  Three and six tiles have no kernel.
// The kernel for few rows is for up to `few_rows` of them and takes `few_strips` at least.
struct Fp4Split { int mt, ns, S; };
inline Fp4Split fp4_split(int M, int N, int K, int n_cu, float join, int most_slices, int few_rows = 16, int few_strips = 1) {
  static const struct { int mt, ns; float us; } tiled[] = {{1, 2, .22f}, {2, 2, .27f}, {4, 2, .40f}, {4, 4, .66f}, {5, 4, .82f}, {7, 4, 1.12f}};
  static const struct { int ns, waves; float us, us_row; } few[] = {{1, 8, 1.f, .07f}, {2, 8, 1.6f, .10f}, {4, 4, 1.f, .06f}};
  const int units = (K + UNIT_K - 1) / UNIT_K, strips = N / 16;
  Fp4Split best = {0, 1, 1};
  float least = 1e30f;
  if (M <= few_rows && fp4_bytes(N, K) < 1u << 31)  // (few rows: gate and up rows in one buffer)
    for (const auto& f : few) {
      if (f.ns < few_strips) continue;
      const float us = .8f + (float)(((strips + f.ns - 1) / f.ns + n_cu - 1) / n_cu) * ((units + f.waves - 1) / f.waves) * (f.us + f.us_row * M);
      if (us < least) { least = us; best = {0, f.ns, 1}; }
    }
  for (const auto& t : tiled) {
    const long long wgs = (long long)((strips + 4 * t.ns - 1) / (4 * t.ns)) * ((M + 16 * t.mt - 1) / (16 * t.mt));
    for (int S = 1; S <= most_slices && S <= units; ++S) {
      if (S > 1 && wgs * S > 2 * n_cu) break;
      const float us = (float)((wgs * S + n_cu - 1) / n_cu) * ((units + S - 1) / S * 2) * t.us + (S > 1 ? join + (float)S * M * N * 1.2e-6f : 0.f);
      if (us < least) { least = us; best = {t.mt, t.ns, S}; }
    }
  }
  return best;
}

// As a call of its own; partial sums of a forward call, whose taker adds them up, in at most `room` floats (S 0: they do not fit);
// and gate/up of a forward call, F columns of either.  Slices that nobody has to join leave the kernel for few rows one or two
// rows of more than 32768 columns (on 256 CUs), four strips a workgroup.
#define FP4_MOST_SLICES 16
#define FP4_PARTS_FEW_ROWS 2
#define FP4_PARTS_FEW_STRIPS 4
inline Fp4Split fp4_split_call(int M, int N, int K, int n_cu) { return fp4_split(M, N, K, n_cu, 7.f, FP4_MOST_SLICES); }
inline Fp4Split fp4_split_parts(int M, int N, int K, int n_cu, size_t room) {
  Fp4Split f = fp4_split(M, N, K, n_cu, 0.f, FP4_MOST_SLICES, FP4_PARTS_FEW_ROWS, FP4_PARTS_FEW_STRIPS);
  while (f.S > 0 && (size_t)f.S * M * N > room) --f.S;
  return f;
}
inline Fp4Split fp4_split_gateup(int M, int F, int K, int n_cu) { return fp4_split(M, 2 * F, K, n_cu, 0.f, 1); }
