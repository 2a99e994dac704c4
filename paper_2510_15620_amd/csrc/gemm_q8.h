// What the kernels of 8-bit products share.
#pragma once

#include "q8.h"

namespace prism {

// What a product of 8-bit rows brings: a scale for each row of A and of W, the distance of the rows in bytes (multiples of 16), and
// the distance of the output's rows in values; of the tiles, by how many slices of K a column tile begins behind the one before it (0: all begin at K's start).
struct Q8Operands {
  const float *sa, *sw;
  uint32_t lda, ldw;
  int64_t ldo;
  int turn;
};

// silu(g) * u in fp32, rounded to 16 bits by its callers.  The division is correctly rounded: a product with the reciprocal
// instruction takes half of this epilogue's arithmetic away (13.8 -> 9.2 thousand cycles of a 256 x 256 tile) and no time where the
// chip is full and at its power limit (24576 x 24576 x 4096: 3350 us, with the division 3337), but is off by
// an ulp more and returns 0 where 1 + e^-g exceeds 2^126, values that bf16 still holds.
__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

// Results of 8-bit products in 16 bits: a NaN (of a row without a scale) stays one, which half's saturation would turn into a number
template <typename T> __device__ __forceinline__ T q8_round(float v) { return from_f32<T>(v); }
template <> __device__ __forceinline__ f16 q8_round<f16>(float v) { return v == v ? from_f32<f16>(v) : (f16)v; }

// Products of few rows, up to 64 (gemm_q8_rows.hip; arguments checked)
int launch_gemm_q8_rows(int epilogue, const prism_q8 &a, const prism_q8 &w, int out_dtype, void *out, int64_t out_stride, hipStream_t s);

}  // namespace prism
