// Products of 8-bit rows (q8.h) on the matrix cores: Y[m][n] = sa[m] sw[n] sum_k a[m][k] w[n][k], with the epilogues of the 16-bit
// products (store, residual add, SwiGLU).
//
// The sum is exact: |a w| <= 2^14 and K < 2^17, so it fits 32-bit integers.  It is converted to fp32 (2^-24), multiplied by sa and then by sw (2^-24 each).
// v_mfma_i32_16x16x64_i8 takes twice the k of the 16-bit instruction from the same bytes in the same cycles, so the kernel is
// the 16-bit products' (gemm_tile.h): a row of K codes is read as K / 2 16-bit values, and in one loop a product takes the time of a 16-bit one of half its K, at the same
// clock (11520 x 4096 x 12288 with residual 480 us, in half with K = 6144 479, both at 1.6 GHz).  What 8 bits change is what a loop half as long shows: the epilogue (gemm_q8.h)
// and how soon weights have to arrive (gen_gemm_kloop.py: BIG; the same product then 411).  11584 x 24576 x 4096 with SwiGLU: 807 to 847 us, 2.75 to 2.89 POP/s, by the chip; of that
// 17 rounds of tiles, matrix pipes busy 70 % of the cycles, a tile's epilogue some 11000 cycles of 90000.
// Codes behind a row's end are zeros up to a multiple of 128, a slice of the loop, so the loop has no tail.
#include "gemm_tile.h"
#include "gemm_q8_plan.h"

namespace prism {

template <typename OT, int EPI>
static int launch_kind(int kind, const int8_t *A, const int8_t *W, void *out, int M, int N, int K, hipStream_t s, const Q8Operands &q, uint32_t lda, uint32_t ldw) {
  switch (kind) {
    case kQ8T256: return launch_tile<OT, 256, 256, 2, 2, EPI, 3>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T224: return launch_tile<OT, 224, 256, 2, 2, EPI, 3>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T192: return launch_tile<OT, 192, 256, 2, 2, EPI, 3>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T160: return launch_tile<OT, 160, 256, 2, 2, EPI, 4>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T128x256: return launch_tile<OT, 128, 256, 2, 2, EPI, 4>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T128: return launch_tile<OT, 128, 128, 2, 2, EPI, 2>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T128Deep: return launch_tile<OT, 128, 128, 2, 2, EPI, 5>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T128x64: return launch_tile<OT, 128, 64, 4, 1, EPI, 3>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T128x64Deep: return launch_tile<OT, 128, 64, 4, 1, EPI, 6>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T64: return launch_tile<OT, 64, 64, 2, 2, EPI, 5>(A, W, out, M, N, K, s, q, lda, ldw);
    case kQ8T32x64: return launch_tile<OT, 32, 64, 1, 1, EPI, 4>(A, W, out, M, N, K, s, q, lda, ldw);
    default: break;
  }
  if constexpr (EPI != PRISM_EPI_SWIGLU) {
    if (kind == kQ8T64x32) return launch_tile<OT, 64, 32, 2, 1, EPI, 7>(A, W, out, M, N, K, s, q, lda, ldw);
    return launch_tile<OT, 32, 32, 2, 2, EPI, 9>(A, W, out, M, N, K, s, q, lda, ldw);
  }
  return PRISM_EUNSUPPORTED;
}

template <typename OT, int EPI>
static int launch_epi(const prism_q8 &a, const prism_q8 &w, void *out, int64_t out_stride, hipStream_t s) {
  constexpr bool kGlu = EPI == PRISM_EPI_SWIGLU;
  constexpr int64_t out_elem = EPI == PRISM_EPI_RESIDUAL || EPI == PRISM_EPI_STORE_F32 ? 4 : 2;
  const int N = w.rows, slices = q8_width(a.cols) / kQ8Slice;
  const Q8Plan p = q8_plan(a.rows, kGlu ? N / 2 : N, slices, kGlu ? kQ8Swiglu : EPI == PRISM_EPI_RESIDUAL ? kQ8Residual : kQ8Store);
  auto rows_on = [&](int kind, int m0, int rows) {
    const Q8Operands q{a.scales + m0, w.scales, out_stride, q8_turn(a.rows, w.stride)};
    return launch_kind<OT, EPI>(kind, a.codes + m0 * a.stride, w.codes, reinterpret_cast<char *>(out) + m0 * out_stride * out_elem, rows, N, slices * BK, s, q, (uint32_t)a.stride,
                                (uint32_t)w.stride);
  };
  if (p.rows_first > 0) PRISM_TRY(rows_on(p.first, 0, p.rows_first));
  return rows_on(p.kind, p.rows_first, a.rows - p.rows_first);
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
  if (q8_few_rows(A->rows, W->rows, A->cols)) return launch_gemm_q8_rows(epilogue, *A, *W, out_dtype, out, out_stride, s);
  const bool half = out_dtype == PRISM_DTYPE_F16;
  switch (epilogue) {
    case PRISM_EPI_STORE: return half ? launch_epi<f16, PRISM_EPI_STORE>(*A, *W, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_STORE>(*A, *W, out, out_stride, s);
    case PRISM_EPI_SWIGLU: return half ? launch_epi<f16, PRISM_EPI_SWIGLU>(*A, *W, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_SWIGLU>(*A, *W, out, out_stride, s);
    case PRISM_EPI_RESIDUAL: return launch_epi<f16, PRISM_EPI_RESIDUAL>(*A, *W, out, out_stride, s);
    default: return launch_epi<f16, PRISM_EPI_STORE_F32>(*A, *W, out, out_stride, s);
  }
}
