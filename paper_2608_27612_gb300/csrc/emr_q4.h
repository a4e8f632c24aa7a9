// The 4-bit weight layout (emr_q4 in emr.h), shared by the packing kernels and the products.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/emr.h"
#include "emr_q8.h"

namespace emr {

// Units of 16 rows x 128 columns follow each other along a row of units: 1024 bytes of codes, 64 of a row after the
// other, and, for each row, the scales of its 128 / group groups. A lane's 16 bytes of codes are what it feeds to m16n8k16
// instructions: lane 4 g + t has rows g and g + 8, and of the w-th 32 columns the word with columns 8 t to 8 t + 7, as pairs
// of columns 16 bits apart; the order of columns in an instruction is such that x is read as it lies.
constexpr int kQ4Rows = 16, kQ4Cols = 128, kQ4Codes = 1024;

__host__ __device__ inline int64_t q4_tiles(int64_t rows) { return (rows + kQ4Rows - 1) / kQ4Rows; }
__host__ __device__ inline int64_t q4_blocks(int64_t cols) { return (cols + kQ4Cols - 1) / kQ4Cols; }
__host__ __device__ inline int q4_unit(int group) { return kQ4Codes + kQ4Rows * 2 * (kQ4Cols / group); }
// Bytes of the scales of rows g and g + 8 in a unit, and where they begin; row g + 8's are the second half.
__host__ __device__ inline int q4_scale_pair(int group) { return 4 * (kQ4Cols / group); }
__host__ __device__ inline int q4_scale_at(int row, int in_block, int group) {
  return kQ4Codes + (row & 7) * q4_scale_pair(group) + ((row >> 3) * (kQ4Cols / group) + in_block) * 2;
}
// Byte of the word with columns 4 q to 4 q + 3 of a block (q < 32) of row r, and the first bit of the first pair.
__host__ __device__ inline int q4_word_at(int row, int q) { return row * 64 + (q >> 1 & 3) * 16 + (q >> 3) * 4; }
__host__ __device__ inline int q4_shift(int q) { return (q & 1) * 8; }
// Four codes in a word: columns 0 and 1 are the first pair, 2 and 3 the second.
__device__ __forceinline__ uint32_t q4_place(int c0, int c1, int c2, int c3, int shift) {
  return (uint32_t(c0 + 8 & 15) | uint32_t(c1 + 8 & 15) << 16 | uint32_t(c2 + 8 & 15) << 4 | uint32_t(c3 + 8 & 15) << 20) << shift;
}

inline bool q4_ok(const emr_q4* q) {
  return q && q->batch > 0 && q->rows > 0 && q->cols > 0 && q->rows <= kQ8MaxDim && q->cols <= kQ8MaxDim &&
         (q->group == 32 || q->group == 64 || q->group == 128) && q->data && reinterpret_cast<uintptr_t>(q->data) % 16 == 0;
}

}  // namespace emr
