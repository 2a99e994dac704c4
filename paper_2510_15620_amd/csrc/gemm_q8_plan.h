// Which kernel a product of 8-bit rows runs on, by estimates of time.  The result does not depend on it: the sums are exact and every kernel rounds what is behind them alike.  (No device code:
// tests compile this file by itself.)
#pragma once

#include <algorithm>
#include <cstdint>

namespace prism {

// A launch deals its tiles over 256 compute units; n = tiles per unit, rounded up.  A tile's time is its slices of 128 codes plus a fixed part (first
// slice, epilogue), and a slice's time depends on how many tiles share the unit: alone it is a chain of latencies, together the matrix pipes, LDS and
// the path to the caches.  The constants are fit to 13 tiles and rings on 256 launches of 17 to 20000 rows, N 64-24576, K 64-12288, all epilogues, weights from memory; the
// pick is on average 0.9 % above the best tile, 22 % at worst (18814 x 256 x 141 residual 13.8 us for 11.3; then 3151 x 2712 x 128 residual 21.9 for 18.7, 18775 x 1037 x 96 residual 46.7
// for 40.2, 2683 x 14939 x 152 residual 98 for 85).
// Large tiles of fewer rows than 256 take a slice in less time, but not in proportion; they pay where their number fills the units better, us on 256, 224, 192, 160, 128 rows by 256 columns and
// on 128 x 128: SwiGLU 600 x 24576 x 4096 91, 85, 77, 70, 67, 71; 1154 x 19456 x 2560 69, 65, 80, 78, 75, 77; 391 x 19456 x 2560 35, 34, 30, 31, 46, 44; stored 1543 x 4096 x 12288 111, 98, 87, 86, 80, 89;
// 3699 x 2560 x 9728 95, 86, 81, 76, 112, 122; 11520 x 4096 x 12288 394, 443, 409, 433, 451, 498.  Two 128 x 128 tiles a unit lead where K is short: one's epilogue runs beside the
// other's loop (10782 x 2048 x 432 SwiGLU 26.4, on 256 x 256 32.5).
struct Q8Tile {
  int bm, bn, occ;                      // tile, workgroups that share a compute unit
  float alone, shared;                  // us per slice: one workgroup on the unit; per workgroup when occ of them share it
  float store, residual, swiglu;        // us per tile
};
enum { kQ8T256, kQ8T224, kQ8T192, kQ8T160, kQ8T128x256, kQ8T128, kQ8T128Deep, kQ8T128x64, kQ8T128x64Deep, kQ8T64, kQ8T32x64, kQ8T64x32, kQ8T32, kQ8Tiles };
static constexpr Q8Tile kQ8Tile[kQ8Tiles] = {
    {256, 256, 1, 1.112f, 1.112f, 11.7f, 22.5f, 9.80f}, {224, 256, 1, 1.009f, 1.009f, 10.6f, 19.9f, 9.18f}, {192, 256, 1, 0.884f, 0.884f, 9.34f, 17.2f, 8.32f},
    {160, 256, 1, 0.818f, 0.818f, 7.74f, 15.2f, 7.48f}, {128, 256, 1, 0.724f, 0.724f, 6.43f, 12.2f, 6.30f},
    {128, 128, 2, 0.661f, 0.462f, 3.83f, 9.26f, 3.80f}, {128, 128, 1, 0.456f, 0.456f, 4.05f, 6.56f, 4.46f},
    {128, 64, 2, 0.307f, 0.325f, 2.55f, 4.58f, 2.91f}, {128, 64, 1, 0.301f, 0.301f, 2.94f, 4.01f, 3.38f},
    {64, 64, 2, 0.212f, 0.219f, 2.05f, 2.78f, 2.55f}, {32, 64, 4, 0.223f, 0.179f, 2.38f, 3.00f, 2.86f},
    {64, 32, 1, 0.160f, 0.160f, 1.91f, 2.16f, 0.f}, {32, 32, 2, 0.064f, 0.107f, 1.74f, 1.89f, 0.f}};
static constexpr float kQ8Launch = 1.3f;   // us

enum Q8Epilogue { kQ8Store, kQ8Residual, kQ8Swiglu };

// (M and cols up to PRISM_MAX_STEP, so that all counts fit 32 bits: their divisions are most of a plan's time on the host, 0.1 us for few rows)
inline float q8_tile_time(const Q8Tile &t, uint32_t M, uint32_t cols, int slices, Q8Epilogue epi) {
  const uint32_t bm = (uint32_t)t.bm, bn = (uint32_t)(epi == kQ8Swiglu ? t.bn / 2 : t.bn), occ = (uint32_t)t.occ;
  const uint32_t tiles = (M + bm - 1) / bm * ((cols + bn - 1) / bn), n = (tiles + 255) / 256, rounds = (n + occ - 1) / occ, last = n - (rounds - 1) * occ;
  // the last of `last` tiles that share a unit shares the caches with few, where it is on few units: 260 tiles of 128 x 128 (1543 x 2501 x 1003) 11.2 us
  const float fill = std::min(1.f, 0.7f + (float)(tiles - (n - 1) * 256) / 256.f), sharing = last > 1 ? (float)(last - 1) + fill : 1.f;
  const float slice = (float)(rounds - 1) * std::max(t.alone, t.shared * (float)occ) + std::max(t.alone, t.shared * sharing);
  return kQ8Launch + (float)slices * slice + (float)rounds * (epi == kQ8Swiglu ? t.swiglu : epi == kQ8Residual ? t.residual : t.store);
}
inline int q8_best_tile(uint32_t M, uint32_t cols, int slices, Q8Epilogue epi, float *time) {
  int at = 0;
  *time = 1e30f;
  for (int k = 0; k < kQ8Tiles; ++k) {
    if (epi == kQ8Swiglu && kQ8Tile[k].bn == 32) continue;              // SwiGLU pairs a gate and an up tile in a wave
    const float t = q8_tile_time(kQ8Tile[k], M, cols, slices, epi);
    if (t < *time) { *time = t; at = k; }
  }
  return at;
}

// What a launch of M rows runs: rows_first rows (whole row tiles, possibly none) on tile `first`, the others on tile `kind` in a launch of their own: the last round
// of large tiles may fill only a few compute units at a whole tile's price.
struct Q8Plan { int rows_first, first, kind; };
inline Q8Plan q8_plan(int M, int cols, int slices, Q8Epilogue epi) {
  float least;
  Q8Plan p{0, 0, q8_best_tile((uint32_t)M, (uint32_t)cols, slices, epi, &least)};
  for (int k = kQ8T256; k <= kQ8T128x256; ++k) {
    const Q8Tile &t = kQ8Tile[k];
    const uint32_t bm = (uint32_t)t.bm, bn = (uint32_t)(epi == kQ8Swiglu ? t.bn / 2 : t.bn), nN = ((uint32_t)cols + bn - 1) / bn, nM = ((uint32_t)M + bm - 1) / bm;
    if (nM * nN <= 256) continue;
    const uint32_t rows = nM * nN / 256 * 256 / nN * bm;                // those that fill whole rounds
    if (rows == 0 || rows >= (uint32_t)M) continue;
    float rest;
    const int kind = q8_best_tile((uint32_t)M - rows, (uint32_t)cols, slices, epi, &rest);
    const float both = q8_tile_time(t, rows, (uint32_t)cols, slices, epi) + rest;
    if (both < 0.98f * least) { least = both; p = {(int)rows, k, kind}; }
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
