// Products of 8-bit rows (q8.h) on the matrix cores: Y[m][n] = sa[m] sw[n] sum_k a[m][k] w[n][k], with the epilogues of the 16-bit
// products (store, residual add, SwiGLU).
//
// The sum is exact: |a w| <= 2^14 and K < 2^17, so it fits 32-bit integers.  It is converted to fp32 (2^-24), multiplied by sa and then by sw (2^-24 each).
// v_mfma_i32_16x16x64_i8 takes twice the k of the 16-bit instruction from the same bytes in the same cycles, so the kernel is
// the 16-bit products' (gemm_tile.h): a row of K codes is read as K / 2 16-bit values.  Codes behind a row's end are zeros up to
// a multiple of 128, a slice of the loop, so the loop has no tail.
#include <algorithm>

#include "gemm_tile.h"

namespace prism {

// ---- which tile a launch uses: the least estimate of time.  The result does not depend on it: sums are exact.
// A launch deals its tiles over 256 compute units; n = tiles per unit, rounded up.  A tile's time is its K slices plus a fixed part (dispatch,
// first slice, epilogue), and a slice's time depends on how many tiles share the unit.
struct Q8Tile {
  int bm, bn, occ;              // tile, workgroups that share a compute unit
  float alone, shared, fixed;   // us per slice of 128 codes: one workgroup on the unit; per workgroup when occ of them share it; us per tile
};
enum { kQ8Tile256, kQ8Tile128, kQ8Tile128Deep, kQ8Tile128x64, kQ8Tile64, kQ8Tile32x64, kQ8Tile64x32, kQ8Tile32, kQ8Tiles };
static constexpr Q8Tile kQ8Tile[kQ8Tiles] = {
    {256, 256, 1, 1.45f, 1.45f, 9.2f}, {128, 128, 2, 0.72f, 0.50f, 4.5f}, {128, 128, 1, 0.52f, 0.52f, 3.4f}, {128, 64, 2, 0.34f, 0.36f, 2.3f},
    {64, 64, 2, 0.204f, 0.204f, 2.1f}, {32, 64, 3, 0.176f, 0.149f, 2.4f}, {64, 32, 1, 0.128f, 0.128f, 2.3f}, {32, 32, 2, 0.106f, 0.083f, 2.6f}};

static double tile_time(const Q8Tile &t, int64_t M, int64_t cols, int slices, bool glu) {
  const int bn = glu ? t.bn / 2 : t.bn;
  const int64_t n = ((M + t.bm - 1) / t.bm * ((cols + bn - 1) / bn) + 255) / 256, full = n / t.occ, rest = n % t.occ;
  const double slice = full * std::max(t.alone, t.shared * t.occ) + (rest ? std::max(t.alone, t.shared * rest) : 0.f);
  return slices * slice + (double)(full + (rest > 0)) * t.fixed;
}
static int best_tile(int64_t M, int64_t cols, int slices, bool glu, double *time) {
  int at = kQ8Tile256;
  *time = tile_time(kQ8Tile[at], M, cols, slices, glu);
  for (int k = 1; k < kQ8Tiles; ++k) {
    if (glu && kQ8Tile[k].bn == 32) continue;              // SwiGLU pairs a gate and an up tile in a wave
    const double t = tile_time(kQ8Tile[k], M, cols, slices, glu);
    if (t < *time) { *time = t; at = k; }
  }
  return at;
}
// rows_big rows (whole tiles of 256, possibly none) run on the largest tile, the others on `kind`: the last round of large tiles may fill only
// a few compute units at a whole tile's price
struct Q8Plan { int rows_big, kind; };
static Q8Plan plan_q8(int M, int cols, int slices, bool glu) {
  double whole, rest;
  const Q8Plan one{0, best_tile(M, cols, slices, glu, &whole)};
  const int64_t nN = cdiv(cols, glu ? 128 : 256), nM = cdiv(M, 256);
  const int big = (int)(nM * nN / 256 * 256 / nN) * 256;
  if (big <= 0 || big >= M) return one;
  const int kind = best_tile(M - big, cols, slices, glu, &rest);
  return kind != kQ8Tile256 && tile_time(kQ8Tile[kQ8Tile256], big, cols, slices, glu) + rest < 0.98 * whole ? Q8Plan{big, kind} : one;
}

template <typename OT, int EPI>
static int launch_kind(int kind, const int8_t *A, const int8_t *W, void *out, int M, int N, int K, hipStream_t s, const Q8Operands &q) {
  switch (kind) {
    case kQ8Tile256: return launch_tile<OT, 256, 256, 2, 2, EPI, 2>(A, W, out, M, N, K, s, q);
    case kQ8Tile128: return launch_tile<OT, 128, 128, 2, 2, EPI, 2>(A, W, out, M, N, K, s, q);
    case kQ8Tile128Deep: return launch_tile<OT, 128, 128, 2, 2, EPI, 4>(A, W, out, M, N, K, s, q);
    case kQ8Tile128x64: return launch_tile<OT, 128, 64, 4, 1, EPI, 3>(A, W, out, M, N, K, s, q);
    case kQ8Tile64: return launch_tile<OT, 64, 64, 2, 2, EPI, 5>(A, W, out, M, N, K, s, q);
    case kQ8Tile32x64: return launch_tile<OT, 32, 64, 1, 1, EPI, 4>(A, W, out, M, N, K, s, q);
    default: break;
  }
  if constexpr (EPI != PRISM_EPI_SWIGLU) {
    if (kind == kQ8Tile64x32) return launch_tile<OT, 64, 32, 2, 1, EPI, 7>(A, W, out, M, N, K, s, q);
    return launch_tile<OT, 32, 32, 2, 2, EPI, 9>(A, W, out, M, N, K, s, q);
  }
  return PRISM_EUNSUPPORTED;
}

template <typename OT, int EPI>
static int launch_epi(const prism_q8 &a, const prism_q8 &w, void *out, int64_t out_stride, hipStream_t s) {
  constexpr bool kGlu = EPI == PRISM_EPI_SWIGLU;
  constexpr size_t out_elem = EPI == PRISM_EPI_RESIDUAL || EPI == PRISM_EPI_STORE_F32 ? 4 : 2;
  const int M = a.rows, N = w.rows, K = q8_width(a.cols) / 2;
  Q8Operands q{a.scales, w.scales, (uint32_t)a.stride, (uint32_t)w.stride, out_stride};
  const Q8Plan p = plan_q8(M, kGlu ? N / 2 : N, K / BK, kGlu);
  if (p.rows_big > 0) PRISM_TRY((launch_kind<OT, EPI>(kQ8Tile256, a.codes, w.codes, out, p.rows_big, N, K, s, q)));
  q.sa += p.rows_big;
  return launch_kind<OT, EPI>(p.kind, a.codes + p.rows_big * a.stride, w.codes, reinterpret_cast<char *>(out) + p.rows_big * out_stride * (int64_t)out_elem,
                              M - p.rows_big, N, K, s, q);
}

}  // namespace prism

using namespace prism;

extern "C" int prism_op_gemm_q8(int32_t epilogue, const prism_q8 *A, const prism_q8 *W, int32_t out_dtype, void *out, int64_t out_stride, void *stream) {
  PRISM_TRY(check_q8(A, "gemm_q8"));
  PRISM_TRY(check_q8(W, "gemm_q8"));
  PRISM_REQUIRE(epilogue >= PRISM_EPI_STORE && epilogue <= PRISM_EPI_STORE_F32, PRISM_EINVAL, "gemm_q8: unknown epilogue %d", epilogue);
  const bool wide = epilogue == PRISM_EPI_RESIDUAL || epilogue == PRISM_EPI_STORE_F32, glu = epilogue == PRISM_EPI_SWIGLU;
  PRISM_REQUIRE(wide ? out_dtype == PRISM_DTYPE_FP32 : is16(out_dtype), PRISM_EINVAL, "gemm_q8: output of type %d with epilogue %d", out_dtype, epilogue);
  PRISM_REQUIRE(A->cols == W->cols, PRISM_EINVAL, "gemm_q8: rows of %d and of %d codes", A->cols, W->cols);
  PRISM_REQUIRE(!glu || W->rows % 2 == 0, PRISM_EUNSUPPORTED, "gemm_q8: SwiGLU of %d rows of weights", W->rows);
  const int64_t cols = glu ? W->rows / 2 : W->rows;
  PRISM_REQUIRE(out_stride >= cols && out_stride <= kQ8MaxStride, PRISM_EINVAL, "gemm_q8: rows of %lld values, %lld apart", (long long)cols, (long long)out_stride);
  // byte offsets within W are 32 bits, with a slice and the loads' bias in hand
  PRISM_REQUIRE(W->rows * W->stride <= ((int64_t)1 << 32) - 8192, PRISM_EUNSUPPORTED, "gemm_q8: weights of %d x %d codes exceed 4 GiB", W->rows, W->cols);
  if (A->rows == 0 || cols == 0) return PRISM_OK;
  PRISM_REQUIRE(out && (uintptr_t)out % (wide ? 4 : 2) == 0, PRISM_EINVAL, "gemm_q8: output missing or not aligned to its values");
  hipStream_t s = (hipStream_t)stream;
  if (gemm_q8_few_rows(A->rows, W->rows, A->cols)) return launch_gemm_q8_rows(epilogue, *A, *W, out_dtype, out, out_stride, s);
  const bool half = out_dtype == PRISM_DTYPE_F16;
  switch (epilogue) {
    case PRISM_EPI_STORE: return half ? launch_epi<f16, PRISM_EPI_STORE>(*A, *W, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_STORE>(*A, *W, out, out_stride, s);
    case PRISM_EPI_SWIGLU: return half ? launch_epi<f16, PRISM_EPI_SWIGLU>(*A, *W, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_SWIGLU>(*A, *W, out, out_stride, s);
    case PRISM_EPI_RESIDUAL: return launch_epi<f16, PRISM_EPI_RESIDUAL>(*A, *W, out, out_stride, s);
    default: return launch_epi<f16, PRISM_EPI_STORE_F32>(*A, *W, out, out_stride, s);
  }
}
