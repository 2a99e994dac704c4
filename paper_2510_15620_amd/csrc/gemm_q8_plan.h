// Which kernel a product of 8-bit rows runs on, by estimates of time.  The result does not depend on it: the sums are exact.  (No device code:
// tests compile this file by itself.)
#pragma once

#include <algorithm>
#include <cstdint>

namespace prism {

// A launch deals its tiles over 256 compute units; n = tiles per unit, rounded up.  A tile's time is its slices of 128 codes plus a fixed part (first
// slice, epilogue), and a slice's time depends on how many tiles share the unit: alone it is a chain of latencies, together the matrix pipes, LDS and
// the path to the caches.  The constants are fit to 11 tiles and rings on 256 launches of 17 to 20000 rows, N 64-24576, K 64-12288, all epilogues, weights from memory; the
// pick is on average 1.1 % above the best tile, 18 % at worst (3151 x 2712 x 128 residual 21.8 us for 18.4; then 2683 x 14939 x 152 residual 98 for 86, 1202 x 1482 x 376 SwiGLU 6.4
// for 5.6, 18814 x 256 x 141 residual 13.7 for 11.9, 1543 x 2501 x 1003 stored 12.6 for 11.1).
// Large tiles of fewer rows than 256 take a slice in less time, but not in proportion (256, 192, 160 rows: 1.13, 0.96, 0.88 us); they pay where
// their number fills the units better: SwiGLU 391 x 19456 x 2560 42.1 (128 x 64), 39.5 (256), 35.0 (160); 777 x 24576 x 4096 102 (128 x 128), 97 (256), 82 (160); residual 3000 x 4096 x 4096
// 57.4 (256), 54.5 (192).  Two 128 x 128 tiles a unit lead where K is short: one's epilogue runs beside the other's loop (10782 x 2048 x 432 SwiGLU 26.4, on 256 x 256 32.5).
struct Q8Tile {
  int bm, bn, occ;                      // tile, workgroups that share a compute unit
  float alone, shared;                  // us per slice: one workgroup on the unit; per workgroup when occ of them share it
  float store, residual, swiglu;        // us per tile
};
enum { kQ8T256, kQ8T192, kQ8T160, kQ8T128, kQ8T128Deep, kQ8T128x64, kQ8T128x64Deep, kQ8T64, kQ8T32x64, kQ8T64x32, kQ8T32, kQ8Tiles };
static constexpr Q8Tile kQ8Tile[kQ8Tiles] = {
    {256, 256, 1, 1.128f, 1.128f, 11.6f, 22.4f, 9.63f}, {192, 256, 1, 0.958f, 0.958f, 8.68f, 17.6f, 7.61f}, {160, 256, 1, 0.884f, 0.884f, 6.98f, 15.7f, 6.79f},
    {128, 128, 2, 0.661f, 0.455f, 3.82f, 9.49f, 3.75f}, {128, 128, 1, 0.437f, 0.437f, 3.95f, 6.56f, 4.41f},
    {128, 64, 2, 0.312f, 0.319f, 2.57f, 4.63f, 2.93f}, {128, 64, 1, 0.297f, 0.297f, 2.94f, 3.98f, 3.37f},
    {64, 64, 2, 0.207f, 0.217f, 2.06f, 2.78f, 2.57f}, {32, 64, 4, 0.218f, 0.176f, 2.41f, 3.10f, 2.88f},
    {64, 32, 1, 0.155f, 0.155f, 1.92f, 2.19f, 0.f}, {32, 32, 2, 0.096f, 0.107f, 1.76f, 1.85f, 0.f}};
static constexpr double kQ8Launch = 1.3;   // us

enum Q8Epilogue { kQ8Store, kQ8Residual, kQ8Swiglu };

inline double q8_tile_time(const Q8Tile &t, int64_t M, int64_t cols, int slices, Q8Epilogue epi) {
  const int bn = epi == kQ8Swiglu ? t.bn / 2 : t.bn;
  const int64_t n = ((M + t.bm - 1) / t.bm * ((cols + bn - 1) / bn) + 255) / 256, full = n / t.occ, rest = n % t.occ;
  const double slice = full * std::max<double>(t.alone, t.shared * t.occ) + (rest ? std::max<double>(t.alone, t.shared * rest) : 0.);
  return kQ8Launch + slices * slice + (double)(full + (rest > 0)) * (epi == kQ8Swiglu ? t.swiglu : epi == kQ8Residual ? t.residual : t.store);
}
inline int q8_best_tile(int64_t M, int64_t cols, int slices, Q8Epilogue epi, double *time) {
  int at = 0;
  *time = 1e30;
  for (int k = 0; k < kQ8Tiles; ++k) {
    if (epi == kQ8Swiglu && kQ8Tile[k].bn == 32) continue;              // SwiGLU pairs a gate and an up tile in a wave
    const double t = q8_tile_time(kQ8Tile[k], M, cols, slices, epi);
    if (t < *time) { *time = t; at = k; }
  }
  return at;
}

// What a launch of M rows runs: rows_first rows (whole row tiles, possibly none) on tile `first`, the others on tile `kind` in a launch of their own: the last round
// of large tiles may fill only a few compute units at a whole tile's price.
struct Q8Plan { int rows_first, first, kind; };
inline Q8Plan q8_plan(int M, int cols, int slices, Q8Epilogue epi) {
  double least;
  Q8Plan p{0, 0, q8_best_tile(M, cols, slices, epi, &least)};
  for (int k = kQ8T256; k <= kQ8T160; ++k) {
    const Q8Tile &t = kQ8Tile[k];
    const int64_t bn = epi == kQ8Swiglu ? t.bn / 2 : t.bn, nN = (cols + bn - 1) / bn, nM = (M + t.bm - 1) / t.bm;
    const int64_t rows = nM * nN / 256 * 256 / nN * t.bm;               // those that fill whole rounds
    if (rows <= 0 || rows >= M) continue;
    double rest;
    const int kind = q8_best_tile(M - rows, cols, slices, epi, &rest);
    const double both = q8_tile_time(t, rows, cols, slices, epi) + rest;
    if (both < 0.98 * least) { least = both; p = {(int)rows, k, kind}; }
  }
  return p;
}

// Launches of few rows that read weights whose rows are a multiple of 4 KiB apart: a column tile begins this many slices of K behind the one before it, and comes round, or all
// compute units would read the same few memory channels at a time.  SwiGLU x 24576 x 4096: 20 rows 24.4 -> 22.1 us, 64 27.2 -> 25.6, 391 70.5 -> 65.0 on 128 x 64 tiles; 391 x 4096 x 4096 15.6 -> 15.1;
// rows 1024 or 2560 codes apart: level.  Many rows' A would leave the caches: 3000 x 4096 x 12288 199 -> 209.
inline int q8_turn(int M, int64_t stride_w) { return M <= 512 && stride_w % 4096 == 0 ? 5 : 0; }

// Whether a product runs on the kernel of few rows (gemm_q8_rows.hip).  Its loads touch 16 cache lines with 64 bytes in each, where the tiles' loads
// into LDS take 8 whole lines, and a compute unit looks up a line in some 4 cycles: nothing for weights, which memory brings at 8 bytes a cycle
// and unit, but every 16 rows of A cost as much again.  us, weights from memory, there / on tiles: 1 x 4096 x 4096 5.5 / 7.0, 16 x 4096 x 4096 6.5 / 7.5,
// 1 x 12288 x 8192 22.9 / 25.1, 16 x 12288 x 8192 28.8 / 24.1, 16 x 512 x 8192 9.0 / 8.2, 1 x 512 x 512 2.0 / 3.1; 32 x 4096 x 1024 3.7 / 4.7, 32 x 12288 x 1024 7.2 / 6.3, 32 x
// 4096 x 4096 8.6 / 8.4; 64 x 2048 x 512 3.5 / 3.9, 64 x 4096 x 1024 4.6 / 4.8, 64 x 512 x 2048 6.3 / 4.2; SwiGLU 24 x 6144 x 1024 4.8 / 5.9, 1 x 24576 x 4096 20.5 / 26.1.
inline bool q8_few_rows(int M, int N, int K) {
  if (M <= 8) return true;
  if (M <= 16) return (int64_t)N * K < 48000000 && (K <= 2048 || N >= 2048);
  return M <= 64 && K <= 1024 && N <= (M <= 32 ? 8192 : 4096);
}

}  // namespace prism
