// Products of a few 8-bit rows (single tokens of some sequences, the last tokens of a pool): every weight is read once, so what counts is
// how many bytes are under way.
//
// Weights go from memory to registers as the matrix instruction wants them, without LDS and without barriers: 16 bytes of k of one of 16 columns a lane.  The waves
// of a workgroup have the same columns and take K's slices of 128 codes by turns (wave w slices w, w + NW, ..), D of them requested ahead; their sums meet in LDS at the
// end, and being integers they are exact in any order.  The rows of A come the same way, out of the caches.  A slice behind the last is requested behind
// the buffer's end, which reads as zeros and moves nothing, so that the loop has no branch that a wait would have to be counted over.
#include "gemm_q8.h"

namespace prism {

typedef __attribute__((ext_vector_type(4))) int i32x4;

template <typename OT, int EPI, int MT, int NT, int NW, int D>
__global__ __launch_bounds__(NW * 64) void gemm_q8_rows_kernel(const int8_t *A, const int8_t *W, int M, int N, int slices, uint32_t bytesA, uint32_t bytesW,
                                                               uint32_t lda, uint32_t ldw, void *out_, Q8Operands q) {
  constexpr bool kGlu = EPI == PRISM_EPI_SWIGLU, kF32 = EPI == PRISM_EPI_RESIDUAL || EPI == PRISM_EPI_STORE_F32;
  constexpr int NO = kGlu ? NT / 2 : NT;                     // tiles of 16 output columns
  constexpr int ITEMS = MT * NO, PER = (ITEMS + NW - 1) / NW; // output tiles; of a wave
  __shared__ i32x4 part[NW][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, group = lane >> 4;
  const int F = kGlu ? N / 2 : N, n0 = blockIdx.x * NO * 16;

  // ---- what a lane reads: rows and columns beyond the matrix are its last ones, whose results nobody stores
  const auto rA = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, (int)bytesA, 0x00027000), rW = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (int)bytesW, 0x00027000);
  uint32_t oA[MT], oW[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) { const int m = i * 16 + row; oA[i] = (uint32_t)(m < M ? m : M - 1) * lda + group * 16u; }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int up = kGlu && j >= NO, c = n0 + (j - up * NO) * 16 + row;
    oW[j] = (uint32_t)((c < F ? c : F - 1) + up * F) * ldw + group * 16u;
  }
  i32x4 a[D][MT][2], w[D][NT][2], acc[MT][NT] = {};
  auto load = [&](int u, int turn) __attribute__((always_inline)) {
    const int s = turn * NW + wave;
    const uint32_t at = (uint32_t)s * 128u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < NT; ++j) w[u][j][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rW, s < slices ? oW[j] + at + h * 64u : 0xfffffff0u, 0, 0));
#pragma unroll
      for (int i = 0; i < MT; ++i) a[u][i][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rA, s < slices ? oA[i] + at + h * 64u : 0xfffffff0u, 0, 0));
    }
  };
#pragma unroll
  for (int u = 0; u < D; ++u) load(u, u);

  // ---- what the epilogue reads, behind the first slices: wave w finishes tiles w, w + NW, ..; a lane has row `row` of A and 4 columns
  typedef f32x4 f32x4_any __attribute__((aligned(4)));
  float sa[PER];
  f32x4 sw[PER][kGlu ? 2 : 1], old[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int t = wave + e * NW, i = t / NO, m = i * 16 + row, c = n0 + t % NO * 16 + group * 4;
    if (t >= ITEMS) continue;
    sa[e] = q.sa[m < M ? m : M - 1];
#pragma unroll
    for (int up = 0; up < (kGlu ? 2 : 1); ++up) {
      const float *s = q.sw + up * F;
      if (c + 4 <= F) sw[e][up] = *reinterpret_cast<const f32x4_any *>(s + c);
      else
        for (int k = 0; k < 4; ++k) sw[e][up][k] = s[c + k < F ? c + k : F - 1];
    }
    if constexpr (EPI == PRISM_EPI_RESIDUAL) {
      const float *o = reinterpret_cast<const float *>(out_) + m * q.ldo + c;
      old[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (m < M && c + 4 <= F) old[e] = *reinterpret_cast<const f32x4_any *>(o);
      else if (m < M)
        for (int k = 0; k < 4; ++k)
          if (c + k < F) old[e][k] = o[k];
    }
  }

  const int turns = (slices + NW - 1) / NW;
  auto use = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][j][h], a[u][i][h], acc[i][j], 0, 0, 0);
  };
  for (int turn = D; turn < turns; turn += D)
#pragma unroll
    for (int u = 0; u < D; ++u) {
      use(u);
      load(u, turn + u);
    }
#pragma unroll
  for (int u = 0; u < D; ++u) use(u);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) part[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int t = wave + e * NW, i = t / NO, j = t % NO, m = i * 16 + row, c = n0 + j * 16 + group * 4;
    if (t >= ITEMS) continue;
    auto total = [&](int tile, const f32x4 &scale) __attribute__((always_inline)) {
      i32x4 sum = part[0][tile][lane];
#pragma unroll
      for (int v = 1; v < NW; ++v) sum += part[v][tile][lane];
      f32x4 y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = q8_scaled(sum[k], sa[e], scale[k]);
      return y;
    };
    f32x4 y = total(i * NT + j, sw[e][0]);
    if constexpr (kGlu) {
      const f32x4 up = total(i * NT + j + NO, sw[e][kGlu ? 1 : 0]);
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = q8_silu_mul(y[k], up[k]);
    }
    if constexpr (EPI == PRISM_EPI_RESIDUAL) y += old[e];
    if (m >= M) continue;
    if constexpr (kF32) {
      float *o = reinterpret_cast<float *>(out_) + m * q.ldo + c;
      if (c + 4 <= F) *reinterpret_cast<f32x4_any *>(o) = y;
      else
        for (int k = 0; k < 4; ++k)
          if (c + k < F) o[k] = y[k];
    } else {
      const auto v = q8_round4<OT>(y);
      typedef decltype(q8_round4<OT>(y)) Quad_any __attribute__((aligned(2)));
      OT *o = reinterpret_cast<OT *>(out_) + m * q.ldo + c;
      if (c + 4 <= F) *reinterpret_cast<Quad_any *>(o) = v;
      else
        for (int k = 0; k < 4; ++k)
          if (c + k < F) o[k] = v[k];
    }
  }
}

template <typename OT, int EPI, int MT, int NT, int NW, int D>
static int launch(const prism_q8 &a, const prism_q8 &w, void *out, int64_t out_stride, hipStream_t s) {
  constexpr int NO = EPI == PRISM_EPI_SWIGLU ? NT / 2 : NT;
  const int F = EPI == PRISM_EPI_SWIGLU ? w.rows / 2 : w.rows, width = q8_width(a.cols);
  const Q8Operands q{a.scales, w.scales, out_stride, 0};
  gemm_q8_rows_kernel<OT, EPI, MT, NT, NW, D><<<cdiv(F, NO * 16), NW * 64, 0, s>>>(a.codes, w.codes, a.rows, w.rows, width / kQ8Slice, (uint32_t)((a.rows - 1) * a.stride + width),
                                                                                  (uint32_t)((w.rows - 1) * w.stride + width), (uint32_t)a.stride, (uint32_t)w.stride, out, q);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

// One column tile a wave (SwiGLU two): more of them in fewer workgroups were slower, 16 x 4096 x 4096 8.6 for two, 14.7 for four.  Slices of K: up to 8, 4 waves; from 32 on, four ahead (1 x
// 24576 x 4096 with SwiGLU 22.3 -> 20.5; on 8 and fewer slices that would ask for slices that are not there, 1 x 1024 x 1024 3.1 -> 3.6).
template <typename OT, int EPI>
static int launch_epi(const prism_q8 &a, const prism_q8 &w, void *out, int64_t out_stride, hipStream_t s) {
  constexpr int NT = EPI == PRISM_EPI_SWIGLU ? 2 : 1;
  const int slices = q8_width(a.cols) / kQ8Slice;
  if (a.rows > 32) return launch<OT, EPI, 4, NT, 4, 2>(a, w, out, out_stride, s);
  if (a.rows > 16) return launch<OT, EPI, 2, NT, 4, 2>(a, w, out, out_stride, s);
  if (slices <= 8) return launch<OT, EPI, 1, NT, 4, 2>(a, w, out, out_stride, s);
  return slices < 32 ? launch<OT, EPI, 1, NT, 8, 2>(a, w, out, out_stride, s) : launch<OT, EPI, 1, NT, 8, 4>(a, w, out, out_stride, s);
}

int launch_gemm_q8_rows(int epilogue, const prism_q8 &a, const prism_q8 &w, int out_dtype, void *out, int64_t out_stride, hipStream_t s) {
  const bool half = out_dtype == PRISM_DTYPE_F16;
  switch (epilogue) {
    case PRISM_EPI_STORE: return half ? launch_epi<f16, PRISM_EPI_STORE>(a, w, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_STORE>(a, w, out, out_stride, s);
    case PRISM_EPI_SWIGLU: return half ? launch_epi<f16, PRISM_EPI_SWIGLU>(a, w, out, out_stride, s) : launch_epi<bf16, PRISM_EPI_SWIGLU>(a, w, out, out_stride, s);
    case PRISM_EPI_RESIDUAL: return launch_epi<f16, PRISM_EPI_RESIDUAL>(a, w, out, out_stride, s);
    default: return launch_epi<f16, PRISM_EPI_STORE_F32>(a, w, out, out_stride, s);
  }
}

}  // namespace prism
