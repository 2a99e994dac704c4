// Rows of 8-bit codes with a scale each (prism_q8), the operands of the products in gemm_q8.hip: made from rows of numbers, made by
// the norm in front of a product, and turned back.
//
// A row x has scale = max|x| / 127 and codes x / scale, rounded to the nearest integer, ties to even.  The norm's rows are n = x r gain with one r a row, which
// cancels in n / scale: code = x gain 127 / max|x gain|, so the sum of squares (for r) and the maximum meet in one reduction and the row is read once.
// All of it is bound by memory; rows stay in registers between the maximum and the codes.
#include <type_traits>

#include "gemm_q8.h"

namespace prism {

static constexpr float kTiny = 1.504632769052528e-36f;       // 2^-119: below it 127 / max leaves fp32, such a row is zeros

// n consecutive values, aligned to one of them only (rows may begin anywhere)
template <typename T, int N> struct Pack {
  typedef T vec __attribute__((ext_vector_type(N)));
  typedef vec any __attribute__((aligned(sizeof(T))));
};
// Values i .. i + N - 1 of a row of n, zeros behind its end.  16 (or 8) bytes that reach over the end are read from further in front and shifted down: one load,
// where a load a value and their waits would hold up the row's other loads
template <typename T, int N> __device__ __forceinline__ typename Pack<T, N>::vec load_row(const T *row, int i, int n) {
  typedef typename Pack<T, N>::vec vec;
  vec v = {};
  if (i + N <= n) v = *reinterpret_cast<const typename Pack<T, N>::any *>(row + i);
  else if (i < n) {
    if (n >= N) {
      typedef std::conditional_t<sizeof(vec) == 16, unsigned __int128, unsigned long long> bits;
      v = *reinterpret_cast<const typename Pack<T, N>::any *>(row + n - N);
      v = __builtin_bit_cast(vec, (bits)(__builtin_bit_cast(bits, v) >> (i + N - n) * (int)sizeof(T) * 8));
    } else {
      for (int e = 0; e < N; ++e)
        if (i + e < n) v[e] = row[i + e];
    }
  }
  return v;
}

__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// As unsigned integers, magnitudes are ordered like their values, infinity behind the finite ones and NaN behind infinity.
// Maximum and sum over a wave, in every lane: within 16 lanes by moves of the vector unit (quads' neighbours, halves mirrored), then by exchanges of 16 and 32 lanes
template <int MOVE> __device__ __forceinline__ unsigned moved(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, MOVE, 0xF, 0xF, false); }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
__device__ __forceinline__ unsigned wave_top(unsigned v) {
  v = larger(v, moved<0xB1>(v));
  v = larger(v, moved<0x4E>(v));
  v = larger(v, moved<0x141>(v));
  v = larger(v, moved<0x140>(v));
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = larger(r[0], r[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return larger(q[0], q[1]);
}
__device__ __forceinline__ float wave_total(float v) {
  v += __uint_as_float(moved<0xB1>(__float_as_uint(v)));
  v += __uint_as_float(moved<0x4E>(__float_as_uint(v)));
  v += __uint_as_float(moved<0x141>(__float_as_uint(v)));
  v += __uint_as_float(moved<0x140>(__float_as_uint(v)));
  return sum_xor32(sum_xor16(v));
}

// Maximum over the T threads of a row (64: of a workgroup's several rows, a wave each), and the sum of NS pieces a thread has.  Piece k of thread t is piece t + k T of the row: 64 pieces
// are summed by a wave, and these sums one after the other in the row's order, so that a row's bits do not depend on how many threads it has, which goes by the number of rows
template <int T, int NS> __device__ __forceinline__ void row_reduce(unsigned &top, float (&piece)[NS > 0 ? NS : 1], float &sum) {
  top = wave_top(top);
#pragma unroll
  for (int k = 0; k < NS; ++k) piece[k] = wave_total(piece[k]);
  if constexpr (T > 64) {
    __shared__ unsigned tops[T / 64];
    __shared__ float sums[NS > 0 ? NS * (T / 64) : 1];
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      tops[w] = top;
#pragma unroll
      for (int k = 0; k < NS; ++k) sums[k * (T / 64) + w] = piece[k];
    }
    __syncthreads();
    top = tops[0];
#pragma unroll
    for (int v = 1; v < T / 64; ++v) top = larger(top, tops[v]);
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < NS * (T / 64); ++v) sum += sums[v];
  } else {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) sum += piece[k];
  }
}
static constexpr int kWaveRows = 4;                          // rows of a workgroup whose rows are a wave's each
template <int T> static constexpr int kGroup = T == 64 ? 64 * kWaveRows : T;

// From a value to its code.  ok: the row has codes at all (finite, not tiny).
// 16-bit rows: x * 127 / max in fp32, corrected by its remainder (all of them times 2^-7, so that nothing overflows), is the correctly rounded quotient; 127 x has at most
// 18 bits, and a quotient of two such numbers that is no tie is further than fp32's spacing from every tie: the codes are exact, ties included.  (x max / 2 in a row is
// a tie, 63.5, and common where numbers have few bits.)  fp32 rows: x times the rounded 127 / max, off by 2^-23 of the quotient at most.
template <bool EXACT> struct Coder {
  float inv, top, back;
  __device__ __forceinline__ explicit Coder(float t) : inv(127.0f / t), top(t * 0.0078125f), back(1.0f / (t * 0.0078125f)) {}
  // the low byte is the code: adding 1.5 * 2^23 rounds to an integer, to even at ties
  __device__ __forceinline__ unsigned operator()(float x) const {
    float q = x * inv;
    if constexpr (EXACT) q = __builtin_fmaf(__builtin_fmaf(-q, top, x * 0.9921875f), back, q);
    return __float_as_uint(q + 12582912.0f);
  }
};
__device__ __forceinline__ unsigned pack_codes(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

// ---- rows of numbers to codes.  A workgroup of T threads per row; NV > 0: up to NV * 16 bytes a thread stay in registers, NV == 0: the row is read twice.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(kGroup<THREADS>) void quantize_q8_kernel(const T *__restrict__ X, int64_t x_stride, int rows, int cols, int width, int8_t *__restrict__ codes,
                                                                      int64_t stride, float *__restrict__ scales) {
  constexpr int N = 16 / sizeof(T);
  typedef typename Pack<T, N>::vec vec;
  const int64_t row = THREADS == 64 ? (int64_t)blockIdx.x * kWaveRows + (threadIdx.x >> 6) : blockIdx.x;
  if (THREADS == 64 && row >= rows) return;
  const int tid = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
  const T *x = X + row * x_stride;
  int8_t *out = codes + row * stride;
  unsigned top = 0;
  float none[1], unused;
  vec keep[NV > 0 ? NV : 1];
  auto look = [&](const vec &v) {
#pragma unroll
    for (int e = 0; e < N; ++e) { const unsigned m = magnitude(to_f32(v[e])); top = top > m ? top : m; }
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) keep[k] = load_row<T, N>(x, (tid + k * THREADS) * N, cols);
#pragma unroll
    for (int k = 0; k < NV; ++k) look(keep[k]);
  } else {
    for (int i = tid * N; i < cols; i += THREADS * N) look(load_row<T, N>(x, i, cols));
  }
  row_reduce<THREADS, 0>(top, none, unused);
  const float t = __uint_as_float(top);
  const bool finite = top < 0x7f800000u, ok = finite && t >= kTiny;
  if (tid == 0) scales[row] = !finite ? __builtin_nanf("") : ok ? t / 127.0f : 0.f;
  const Coder<(sizeof(T) == 2)> code(ok ? t : 1.0f);
  auto emit = [&](int i, const vec &v) {
    if (i >= width) return;
    unsigned w[N / 4];
#pragma unroll
    for (int e = 0; e < N; e += 4)
      w[e / 4] = ok ? pack_codes(code(to_f32(v[e])), code(to_f32(v[e + 1])), code(to_f32(v[e + 2])), code(to_f32(v[e + 3]))) : 0u;
    if constexpr (N == 8) *reinterpret_cast<uint2 *>(out + i) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<unsigned *>(out + i) = w[0];
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) emit((tid + k * THREADS) * N, keep[k]);
  } else {
    for (int i = tid * N; i < width; i += THREADS * N) emit(i, load_row<T, N>(x, i, cols));
  }
}

// ---- the norm.  X += add (where given, rounded once to fp32); codes of X gain / sqrt(mean X^2 + eps)
struct NormArgs {
  float *X;
  const void *add, *gain;
  int x_stride, add_stride, rows, cols, width;
  float eps;
  int8_t *codes;
  int64_t stride;
  float *scales;
};
struct NoAdd {};
template <typename TD, typename TG, int THREADS, int NV>
__global__ __launch_bounds__(kGroup<THREADS>) void rmsnorm_q8_kernel(float *X, const void *add, const void *gain_, int x_stride, int add_stride, int rows, int cols,
                                                                     int width, float eps, int8_t *codes, int64_t stride, float *scales) {
  constexpr bool kAdd = !__is_same(TD, NoAdd);
  const int64_t row = THREADS == 64 ? (int64_t)blockIdx.x * kWaveRows + (threadIdx.x >> 6) : blockIdx.x;
  if (THREADS == 64 && row >= rows) return;
  const int tid = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
  float *x = X + row * x_stride;
  const TG *gain = reinterpret_cast<const TG *>(gain_);
  int8_t *out = codes + row * stride;
  unsigned top = 0;
  constexpr int NS = NV > 0 ? NV : 1;
  float squares[NS] = {}, ss;
  f32x4 keep[NS];
  // x gain of four values; x with the addition is stored, its squares are summed
  auto step = [&](int i, f32x4 v, const auto &d, const typename Pack<TG, 4>::vec &g, float &squares) {
    if constexpr (kAdd) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += to_f32(d[e]);
      if (i + 4 <= cols) *reinterpret_cast<typename Pack<float, 4>::any *>(x + i) = v;
      else
        for (int e = 0; e < 4; ++e)
          if (i + e < cols) x[i + e] = v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      squares += v[e] * v[e];
      v[e] *= to_f32(g[e]);
      const unsigned m = magnitude(v[e]);
      top = top > m ? top : m;
    }
    return v;
  };
  auto load_add = [&](int i) {
    if constexpr (kAdd) return load_row<TD, 4>(reinterpret_cast<const TD *>(add) + row * add_stride, i, cols);
    else return 0;
  };
  if constexpr (NV > 0) {
    decltype(load_add(0)) d[NV];
    typename Pack<TG, 4>::vec g[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = (tid + k * THREADS) * 4;
      keep[k] = load_row<float, 4>(x, i, cols);
      d[k] = load_add(i);
      g[k] = load_row<TG, 4>(gain, i, cols);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) keep[k] = step((tid + k * THREADS) * 4, keep[k], d[k], g[k], squares[k]);
  } else {
    for (int i = tid * 4; i < cols; i += THREADS * 4) step(i, load_row<float, 4>(x, i, cols), load_add(i), load_row<TG, 4>(gain, i, cols), squares[0]);
  }
  row_reduce<THREADS, NS>(top, squares, ss);
  const float t = __uint_as_float(top);
  bool finite = top < 0x7f800000u && ss < __builtin_inff();
  auto largest = [&] { return t * (1.0f / sqrtf(ss / (float)cols + eps)); };      // of the normed row
  // (r is 10^15 at most, eps being 10^-30 at least: the normed values of ordinary rows are known to be finite without it)
  if (t >= 0x1p78f) finite = finite && largest() < __builtin_inff();
  const bool ok = finite && t >= kTiny;
  if (tid == 0) scales[row] = !finite ? __builtin_nanf("") : ok ? largest() / 127.0f : 0.f;
  const Coder<false> code(ok ? t : 1.0f);
  auto emit = [&](int i, const f32x4 &v) {
    if (i < width) *reinterpret_cast<unsigned *>(out + i) = ok ? pack_codes(code(v[0]), code(v[1]), code(v[2]), code(v[3])) : 0u;
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) emit((tid + k * THREADS) * 4, keep[k]);
  } else {
    // each thread reads back what it stored itself
    for (int i = tid * 4; i < width; i += THREADS * 4) {
      f32x4 v = load_row<float, 4>(x, i, cols);
      const auto g = load_row<TG, 4>(gain, i, cols);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= to_f32(g[e]);
      emit(i, v);
    }
  }
}

// ---- back to numbers: code * scale, rounded once more to 16 bits.  256 threads take 8 codes each, of 256 / lanes rows; where these are too few workgroups for the
// chip, each of several takes a part of the columns (7 x 12288 3.7 -> 2.6 us)
template <typename T>
__global__ __launch_bounds__(256) void dequantize_q8_kernel(const int8_t *__restrict__ codes, int64_t stride, const float *__restrict__ scales, int rows, int cols, int lanes,
                                                            T *__restrict__ out, int64_t out_stride) {
  const int64_t row = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
  if (row >= rows) return;
  const float s = scales[row];
  const int8_t *in = codes + row * stride;
  T *o = out + row * out_stride;
  for (int i = (blockIdx.y * lanes + threadIdx.x % lanes) * 8; i < cols; i += gridDim.y * lanes * 8) {
    const uint2 c = *reinterpret_cast<const uint2 *>(in + i);
    f32x4 x[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e / 4][e % 4] = (float)(int8_t)((e < 4 ? c.x : c.y) >> (e & 3) * 8) * s;
    const auto lo = q8_round4<T>(x[0]), hi = q8_round4<T>(x[1]);
    const typename Pack<T, 8>::vec v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    if (i + 8 <= cols) *reinterpret_cast<typename Pack<T, 8>::any *>(o + i) = v;
    else
      for (int e = 0; e < 8; ++e)
        if (i + e < cols) o[i + e] = v[e];
  }
}

int check_q8(const prism_q8 *q, const char *who) {
  PRISM_REQUIRE(q, PRISM_EINVAL, "%s: no 8-bit rows", who);
  PRISM_REQUIRE(q->rows >= 0 && q->rows <= PRISM_MAX_STEP && q->cols > 0 && q->cols <= kQ8MaxCols, PRISM_EINVAL, "%s: %d rows of %d codes", who, q->rows, q->cols);
  PRISM_REQUIRE(q->stride >= q8_width(q->cols) && q->stride <= kQ8MaxStride && q->stride % 16 == 0, PRISM_EINVAL,
                "%s: rows of %d codes are %d bytes apart at least, a multiple of 16", who, q->cols, q8_width(q->cols));
  PRISM_REQUIRE(q->rows == 0 || (q->codes && q->scales && (uintptr_t)q->codes % 16 == 0 && (uintptr_t)q->scales % 4 == 0), PRISM_EINVAL,
                "%s: codes or scales missing or not aligned", who);
  return PRISM_OK;
}

// Threads of a row, from its 16-byte pieces and the number of rows.  Few rows are a chain of latencies, so a thread takes one piece, of long rows two or four; many rows fill the
// chip anyway, and a row of few pieces in many threads is mostly the meeting of its waves.  us at 64, 128, 256, 512, 1024 threads: norm of 24 x 4096 11.1, 4.3, 3.5, 3.2, 3.2; 1 x
// 12288 24.6, 13.4, 8.2, 4.6, 4.3; 16000 x 500 22.0, 22.7, 27.3, 42.9, 74.3; 16000 x 1003 39.8, 37.3, 40.0, 56.0, 94.4; 16000 x 4096 155, 126, 122, 122, 121; codes of bf16 24 x 12288
// 13.8, 7.4, 3.7, 3.3, 3.3; 60000 x 1003 35.3, 46.7, 59.3, 94.0, 167; 4099 x 12288 38.4, 45.6, 27.2, 27.1, 26.4.
static int row_threads(int pieces, int rows) {
  if (rows < 1024) return pieces <= 64 ? 64 : pieces <= 128 ? 128 : pieces <= 256 ? 256 : pieces <= 1024 ? 512 : 1024;
  return pieces <= 128 ? 64 : pieces <= 256 ? 128 : pieces <= 1024 ? 256 : pieces <= 2048 ? 512 : 1024;
}
// Calls run(threads, pieces of a thread that stay in registers, 0: the row is read twice), both as types, and the grid
template <typename F> static void for_rows(int pieces, int rows, F &&run) {
  const int threads = row_threads(pieces, rows), per = (pieces + threads - 1) / threads;
  auto with = [&](auto t) {
    constexpr int T = decltype(t)::value;
    const int grid = T == 64 ? cdiv(rows, kWaveRows) : rows;
    if constexpr (T < 1024)
      if (per <= 1) return run(t, std::integral_constant<int, 1>{}, grid);
    if (per <= 2) return run(t, std::integral_constant<int, 2>{}, grid);
    if constexpr (T >= 256)
      if (per <= 4) return run(t, std::integral_constant<int, 4>{}, grid);
    if constexpr (T == 1024) run(t, std::integral_constant<int, 0>{}, grid);
  };
  if (threads == 64) with(std::integral_constant<int, 64>{});
  else if (threads == 128) with(std::integral_constant<int, 128>{});
  else if (threads == 256) with(std::integral_constant<int, 256>{});
  else if (threads == 512) with(std::integral_constant<int, 512>{});
  else with(std::integral_constant<int, 1024>{});
}

template <typename T> static void launch_quantize(const void *X, int64_t x_stride, const prism_q8 &q, hipStream_t s) {
  const int width = q8_width(q.cols);
  for_rows(width / (16 / (int)sizeof(T)), q.rows, [&](auto t, auto nv, int grid) {
    quantize_q8_kernel<T, decltype(t)::value, decltype(nv)::value>
        <<<grid, kGroup<decltype(t)::value>, 0, s>>>((const T *)X, x_stride, q.rows, q.cols, width, q.codes, q.stride, q.scales);
  });
}

template <typename TD, typename TG> static void launch_norm(const NormArgs &a, int rows, hipStream_t s) {
  for_rows(a.width / 4, rows, [&](auto t, auto nv, int grid) {
    rmsnorm_q8_kernel<TD, TG, decltype(t)::value, decltype(nv)::value><<<grid, kGroup<decltype(t)::value>, 0, s>>>(
        a.X, a.add, a.gain, a.x_stride, a.add_stride, a.rows, a.cols, a.width, a.eps, a.codes, a.stride, a.scales);
  });
}
template <typename TD> static void launch_norm_gain(int gain_dtype, const NormArgs &a, int rows, hipStream_t s) {
  if (gain_dtype == PRISM_DTYPE_FP32) launch_norm<TD, float>(a, rows, s);
  else if (gain_dtype == PRISM_DTYPE_BF16) launch_norm<TD, bf16>(a, rows, s);
  else launch_norm<TD, f16>(a, rows, s);
}

static bool known(int dtype) { return dtype == PRISM_DTYPE_FP32 || is16(dtype); }

}  // namespace prism

using namespace prism;

extern "C" int prism_op_quantize_q8(int32_t dtype, const void *X, int64_t x_stride, const prism_q8 *out, void *stream) {
  PRISM_TRY(check_q8(out, "quantize_q8"));
  PRISM_REQUIRE(known(dtype), PRISM_EINVAL, "quantize_q8: unknown dtype %d", dtype);
  PRISM_REQUIRE(x_stride >= out->cols && x_stride <= kQ8MaxStride, PRISM_EINVAL, "quantize_q8: rows of %d values, %lld apart", out->cols, (long long)x_stride);
  if (out->rows == 0) return PRISM_OK;
  PRISM_REQUIRE(X && (uintptr_t)X % dtype_size(dtype) == 0, PRISM_EINVAL, "quantize_q8: input missing or not aligned to its values");
  hipStream_t s = (hipStream_t)stream;
  if (dtype == PRISM_DTYPE_FP32) launch_quantize<float>(X, x_stride, *out, s);
  else if (dtype == PRISM_DTYPE_BF16) launch_quantize<bf16>(X, x_stride, *out, s);
  else launch_quantize<f16>(X, x_stride, *out, s);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

extern "C" int prism_op_dequantize_q8(const prism_q8 *q, int32_t dtype, void *out, int64_t out_stride, void *stream) {
  PRISM_TRY(check_q8(q, "dequantize_q8"));
  PRISM_REQUIRE(known(dtype), PRISM_EINVAL, "dequantize_q8: unknown dtype %d", dtype);
  PRISM_REQUIRE(out_stride >= q->cols && out_stride <= kQ8MaxStride, PRISM_EINVAL, "dequantize_q8: rows of %d values, %lld apart", q->cols, (long long)out_stride);
  if (q->rows == 0) return PRISM_OK;
  PRISM_REQUIRE(out && (uintptr_t)out % dtype_size(dtype) == 0, PRISM_EINVAL, "dequantize_q8: output missing or not aligned to its values");
  int lanes = 8;
  while (lanes < 256 && lanes * 8 < q->cols) lanes *= 2;
  const int groups = cdiv(q->rows, 256 / lanes);
  const dim3 grid(groups, groups < 1024 ? cdiv(q->cols, lanes * 8) : 1);
  auto run = [&](auto *o) { dequantize_q8_kernel<<<grid, 256, 0, (hipStream_t)stream>>>(q->codes, q->stride, q->scales, q->rows, q->cols, lanes, o, out_stride); };
  if (dtype == PRISM_DTYPE_FP32) run((float *)out);
  else if (dtype == PRISM_DTYPE_BF16) run((bf16 *)out);
  else run((f16 *)out);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

extern "C" int prism_op_rmsnorm_q8(float *X, int64_t x_stride, int32_t add_dtype, const void *add, int64_t add_stride, int32_t gain_dtype, const void *gain, float eps,
                                   const prism_q8 *out, void *stream) {
  PRISM_TRY(check_q8(out, "rmsnorm_q8"));
  PRISM_REQUIRE(known(gain_dtype) && (!add || known(add_dtype)), PRISM_EINVAL, "rmsnorm_q8: unknown dtype %d, %d", gain_dtype, add_dtype);
  PRISM_REQUIRE(eps >= 1e-30f && eps < 1e30f, PRISM_EINVAL, "rmsnorm_q8: eps of %g", eps);
  PRISM_REQUIRE(x_stride >= out->cols && x_stride <= kQ8MaxStride && (!add || (add_stride >= out->cols && add_stride <= kQ8MaxStride)), PRISM_EINVAL,
                "rmsnorm_q8: rows of %d values, %lld and %lld apart", out->cols, (long long)x_stride, (long long)add_stride);
  if (out->rows == 0) return PRISM_OK;
  PRISM_REQUIRE(X && gain && (uintptr_t)X % 4 == 0 && (uintptr_t)gain % dtype_size(gain_dtype) == 0 && (!add || (uintptr_t)add % dtype_size(add_dtype) == 0), PRISM_EINVAL,
                "rmsnorm_q8: X or gain missing, or one not aligned to its values");
  const NormArgs a{X, add, gain, (int)x_stride, (int)add_stride, out->rows, out->cols, q8_width(out->cols), eps, out->codes, out->stride, out->scales};
  hipStream_t s = (hipStream_t)stream;
  if (!add) launch_norm_gain<NoAdd>(gain_dtype, a, out->rows, s);
  else if (add_dtype == PRISM_DTYPE_FP32) launch_norm_gain<float>(gain_dtype, a, out->rows, s);
  else if (add_dtype == PRISM_DTYPE_BF16) launch_norm_gain<bf16>(gain_dtype, a, out->rows, s);
  else launch_norm_gain<f16>(gain_dtype, a, out->rows, s);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}
