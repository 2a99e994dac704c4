// What the kernels of 8-bit products share.
#pragma once

#include "q8.h"

namespace prism {

// What a product of 8-bit rows brings: a scale for each row of A and of W, and the distance of the output's rows in values; of the tiles, by how many slices of K a column tile begins behind the one before it (0: all begin at K's start).
struct Q8Operands {
  const float *sa, *sw;
  int64_t ldo;
  int turn;
};

// A sum times its scales, each product rounded: never one operation with the addition to a stream behind it, which the kernel of few rows has in the same registers
// and the tiles behind LDS.  A quarter of the stream's values would differ in their last bit between the two, and a row's bits go by the row and W alone.
__device__ __forceinline__ float q8_scaled(int sum, float sa, float sw) {
#pragma clang fp contract(off)
  return (float)sum * sa * sw;
}

// silu(g) * u of the 8-bit products, off by 6.5 + 1.5 |g| in 2^-24 (exponential, its argument, sum, reciprocal, two products).  Their loops are half as long
// as the 16-bit ones, so that the epilogue is a quarter of a tile of K = 4096, and a division's ten instructions show (with the two-at-a-time rounding below, us: 11520 x 24576 x 4096
// 895 -> 847, x 1024 355 -> 313; the rounding alone, stored 11520 x 12288 x 4096 450 -> 432).  Where 1 + e^-g
// exceeds 2^126 the reciprocal is 0: the result is then below 10^-36 |u|.
__device__ __forceinline__ float q8_silu_mul(float g, float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

// Results of 8-bit products in 16 bits: rounded to nearest, half saturated.  A NaN (of a row without a scale) stays one; gfx950's minimum and maximum of
// three keep it, and take two values at a time.
template <typename T> __device__ __forceinline__ auto q8_round4(const f32x4 &v) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 r = __builtin_convertvector(v, T4);
  if constexpr (__is_same(T, f16)) {
    constexpr f16 top = (f16)65504.0f;
    const T4 hi = {top, top, top, top};
    r = __builtin_elementwise_minimum(__builtin_elementwise_maximum(r, -hi), hi);
  }
  return r;
}

// Products of few rows, up to 64 (gemm_q8_rows.hip; arguments checked)
int launch_gemm_q8_rows(int epilogue, const prism_q8 &a, const prism_q8 &w, int out_dtype, void *out, int64_t out_stride, hipStream_t s);

}  // namespace prism
