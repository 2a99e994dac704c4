// 8-bit rows: what their makers (q8.hip) and readers (gemm_q8.hip) share.
#pragma once

#include "common.h"

namespace prism {

static constexpr int kQ8Slice = 128;                  // codes that a step of a product reads of a row: rows are zeros from cols up to a multiple of it
static constexpr int kQ8MaxCols = 131071;             // 2^14 cols stays below 2^31
static constexpr int64_t kQ8MaxStride = 1 << 23;      // of rows, in values: 256 rows of four-byte values stay below 2^33, of 32 below 2^30

__host__ __device__ inline int q8_width(int cols) { return (cols + kQ8Slice - 1) / kQ8Slice * kQ8Slice; }

int check_q8(const prism_q8 *q, const char *who);

}  // namespace prism
