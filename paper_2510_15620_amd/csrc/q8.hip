// Rows of 8-bit codes with a scale each (prism_q8), the operands of the products in gemm_q8.hip: made from rows of numbers, made by
// the norm in front of a product, and turned back.
//
// A row x has scale = max|x| / 127 and codes x / scale, rounded to the nearest integer, ties to even.  The norm's rows are n = x r gain with one r a row, which
// cancels in n / scale: code = x gain 127 / max|x gain|, so the sum of squares (for r) and the maximum meet in one reduction and the row is read once.
// All of it is bound by memory; rows stay in registers between the maximum and the codes.
#include "gemm_q8.h"

namespace prism {

static constexpr float kTiny = 1.504632769052528e-36f;       // 2^-119: below it 127 / max leaves fp32, such a row is zeros

// n consecutive values, aligned to one of them only (rows may begin anywhere)
template <typename T, int N> struct Pack {
  typedef T vec __attribute__((ext_vector_type(N)));
  typedef vec any __attribute__((aligned(sizeof(T))));
};
// values i .. i + N - 1 of a row of n, zeros behind its end
template <typename T, int N> __device__ __forceinline__ typename Pack<T, N>::vec load_row(const T *row, int i, int n) {
  typename Pack<T, N>::vec v = {};
  if (i + N <= n) v = *reinterpret_cast<const typename Pack<T, N>::any *>(row + i);
  else
    for (int e = 0; e < N; ++e)
      if (i + e < n) v[e] = row[i + e];
  return v;
}

__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// As unsigned integers, magnitudes are ordered like their values, infinity behind the finite ones and NaN behind infinity
__device__ __forceinline__ unsigned wave_max_u(unsigned v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { const unsigned w = __shfl_xor(v, o, 64); v = v > w ? v : w; }
  return v;
}

// Maximum (and sum) over a workgroup of T threads
template <int T> __device__ __forceinline__ void block_reduce(unsigned &top, float &sum) {
  __shared__ unsigned tops[T / 64];
  __shared__ float sums[T / 64];
  top = wave_max_u(top);
  sum = wave_sum(sum);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) { tops[threadIdx.x >> 6] = top; sums[threadIdx.x >> 6] = sum; }
    __syncthreads();
    top = tops[0]; sum = sums[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) { top = top > tops[w] ? top : tops[w]; sum += sums[w]; }
  }
}

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
__global__ __launch_bounds__(THREADS) void quantize_q8_kernel(const T *__restrict__ X, int64_t x_stride, int cols, int width, int8_t *__restrict__ codes, int64_t stride,
                                                              float *__restrict__ scales) {
  constexpr int N = 16 / sizeof(T);
  typedef typename Pack<T, N>::vec vec;
  const int64_t row = blockIdx.x;
  const T *x = X + row * x_stride;
  int8_t *out = codes + row * stride;
  unsigned top = 0;
  float unused = 0.f;
  vec keep[NV > 0 ? NV : 1];
  auto look = [&](const vec &v) {
#pragma unroll
    for (int e = 0; e < N; ++e) { const unsigned m = magnitude(to_f32(v[e])); top = top > m ? top : m; }
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) keep[k] = load_row<T, N>(x, (threadIdx.x + k * THREADS) * N, cols);
#pragma unroll
    for (int k = 0; k < NV; ++k) look(keep[k]);
  } else {
    for (int i = threadIdx.x * N; i < cols; i += THREADS * N) look(load_row<T, N>(x, i, cols));
  }
  block_reduce<THREADS>(top, unused);
  const float t = __uint_as_float(top);
  const bool finite = top < 0x7f800000u, ok = finite && t >= kTiny;
  if (threadIdx.x == 0) scales[row] = !finite ? __builtin_nanf("") : ok ? t / 127.0f : 0.f;
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
    for (int k = 0; k < NV; ++k) emit((threadIdx.x + k * THREADS) * N, keep[k]);
  } else {
    for (int i = threadIdx.x * N; i < width; i += THREADS * N) emit(i, load_row<T, N>(x, i, cols));
  }
}

// ---- the norm.  X += add (where given, rounded once to fp32); codes of X gain / sqrt(mean X^2 + eps)
struct NormArgs {
  float *X;
  const void *add, *gain;
  int64_t x_stride, add_stride, stride;
  int8_t *codes;
  float *scales;
  int cols, width;
  float eps;
};
struct NoAdd {};
template <typename TD, typename TG, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void rmsnorm_q8_kernel(NormArgs a) {
  constexpr bool kAdd = !__is_same(TD, NoAdd);
  const int64_t row = blockIdx.x;
  float *x = a.X + row * a.x_stride;
  const TG *gain = reinterpret_cast<const TG *>(a.gain);
  int8_t *out = a.codes + row * a.stride;
  unsigned top = 0;
  float ss = 0.f;
  f32x4 keep[NV > 0 ? NV : 1];
  // x gain of four values; x with the addition is stored, its squares are summed
  auto step = [&](int i, f32x4 v, const auto &d, const typename Pack<TG, 4>::vec &g) {
    if constexpr (kAdd) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += to_f32(d[e]);
      if (i + 4 <= a.cols) *reinterpret_cast<typename Pack<float, 4>::any *>(x + i) = v;
      else
        for (int e = 0; e < 4; ++e)
          if (i + e < a.cols) x[i + e] = v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ss += v[e] * v[e];
      v[e] *= to_f32(g[e]);
      const unsigned m = magnitude(v[e]);
      top = top > m ? top : m;
    }
    return v;
  };
  auto load_add = [&](int i) {
    if constexpr (kAdd) return load_row<TD, 4>(reinterpret_cast<const TD *>(a.add) + row * a.add_stride, i, a.cols);
    else return 0;
  };
  if constexpr (NV > 0) {
    decltype(load_add(0)) d[NV];
    typename Pack<TG, 4>::vec g[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = (threadIdx.x + k * THREADS) * 4;
      keep[k] = load_row<float, 4>(x, i, a.cols);
      d[k] = load_add(i);
      g[k] = load_row<TG, 4>(gain, i, a.cols);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) keep[k] = step((threadIdx.x + k * THREADS) * 4, keep[k], d[k], g[k]);
  } else {
    for (int i = threadIdx.x * 4; i < a.cols; i += THREADS * 4) step(i, load_row<float, 4>(x, i, a.cols), load_add(i), load_row<TG, 4>(gain, i, a.cols));
  }
  block_reduce<THREADS>(top, ss);
  const float t = __uint_as_float(top);
  const bool finite = top < 0x7f800000u && ss < __builtin_inff(), ok = finite && t >= kTiny;
  if (threadIdx.x == 0) {
    const float r = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
    a.scales[row] = !finite ? __builtin_nanf("") : ok ? t * r / 127.0f : 0.f;
  }
  const Coder<false> code(ok ? t : 1.0f);
  auto emit = [&](int i, const f32x4 &v) {
    if (i < a.width) *reinterpret_cast<unsigned *>(out + i) = ok ? pack_codes(code(v[0]), code(v[1]), code(v[2]), code(v[3])) : 0u;
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) emit((threadIdx.x + k * THREADS) * 4, keep[k]);
  } else {
    // each thread reads back what it stored itself
    for (int i = threadIdx.x * 4; i < a.width; i += THREADS * 4) {
      f32x4 v = load_row<float, 4>(x, i, a.cols);
      const auto g = load_row<TG, 4>(gain, i, a.cols);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= to_f32(g[e]);
      emit(i, v);
    }
  }
}

// ---- back to numbers: code * scale, rounded once more to 16 bits.  256 threads take 8 codes each, of 256 / lanes rows
template <typename T>
__global__ __launch_bounds__(256) void dequantize_q8_kernel(const int8_t *__restrict__ codes, int64_t stride, const float *__restrict__ scales, int rows, int cols, int lanes,
                                                            T *__restrict__ out, int64_t out_stride) {
  const int64_t row = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
  if (row >= rows) return;
  const float s = scales[row];
  const int8_t *in = codes + row * stride;
  T *o = out + row * out_stride;
  for (int i = (threadIdx.x % lanes) * 8; i < cols; i += lanes * 8) {
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

template <typename T> static void launch_quantize(const void *X, int64_t x_stride, const prism_q8 &q, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const int width = q8_width(q.cols), per = (width + 256 * N - 1) / (256 * N);
  auto run = [&](auto kern, int threads) { kern<<<q.rows, threads, 0, s>>>((const T *)X, x_stride, q.cols, width, q.codes, q.stride, q.scales); };
  if (width <= 64 * N) run(quantize_q8_kernel<T, 64, 1>, 64);
  else if (per <= 1) run(quantize_q8_kernel<T, 256, 1>, 256);
  else if (per <= 2) run(quantize_q8_kernel<T, 256, 2>, 256);
  else if (per <= 4) run(quantize_q8_kernel<T, 256, 4>, 256);
  else if (per <= 8) run(quantize_q8_kernel<T, 256, 8>, 256);
  else run(quantize_q8_kernel<T, 256, 0>, 256);
}

template <typename TD, typename TG> static void launch_norm(const NormArgs &a, int rows, hipStream_t s) {
  const int per = (a.width + 1023) / 1024;
  if (a.width <= 256) rmsnorm_q8_kernel<TD, TG, 64, 1><<<rows, 64, 0, s>>>(a);
  else if (per <= 1) rmsnorm_q8_kernel<TD, TG, 256, 1><<<rows, 256, 0, s>>>(a);
  else if (per <= 2) rmsnorm_q8_kernel<TD, TG, 256, 2><<<rows, 256, 0, s>>>(a);
  else if (per <= 4) rmsnorm_q8_kernel<TD, TG, 256, 4><<<rows, 256, 0, s>>>(a);
  else if (per <= 8) rmsnorm_q8_kernel<TD, TG, 256, 8><<<rows, 256, 0, s>>>(a);
  else rmsnorm_q8_kernel<TD, TG, 256, 0><<<rows, 256, 0, s>>>(a);
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
  const int grid = cdiv(q->rows, 256 / lanes);
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
  const NormArgs a{X, add, gain, x_stride, add_stride, out->stride, out->codes, out->scales, out->cols, q8_width(out->cols), eps};
  hipStream_t s = (hipStream_t)stream;
  if (!add) launch_norm_gain<NoAdd>(gain_dtype, a, out->rows, s);
  else if (add_dtype == PRISM_DTYPE_FP32) launch_norm_gain<float>(gain_dtype, a, out->rows, s);
  else if (add_dtype == PRISM_DTYPE_BF16) launch_norm_gain<bf16>(gain_dtype, a, out->rows, s);
  else launch_norm_gain<f16>(gain_dtype, a, out->rows, s);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}
