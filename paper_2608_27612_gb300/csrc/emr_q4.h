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

// Two codes, 16 bits apart, as 16-bit floats: 1024 + q or 128 + q with q = code + 8, and the rest taken off.
template <bool kHalf>
__device__ __forceinline__ uint32_t codes(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "r"(0x000f000fu), "r"(kHalf ? 0x64006400u : 0x43004300u));  // (w & mask) | ones
  if (kHalf) asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(r) : "r"(0x64086408u));
  else asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x43084308u));
  return r;
}
// Two 32-bit values as pairs of bfloat16: a part of each takes the next 8 bits of its fraction. An infinity is the first part
// alone, a NaN each.
__device__ __forceinline__ void split_pair(float v0, float v1, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const uint32_t a = __float_as_uint(v0), b = __float_as_uint(v1);
  hi = __byte_perm(a, b, 0x7632);
  const float left0 = fabsf(v0) == INFINITY ? 0.f : v0 - __uint_as_float(a & 0xffff0000u);
  const float left1 = fabsf(v1) == INFINITY ? 0.f : v1 - __uint_as_float(b & 0xffff0000u);
  const uint32_t c = __float_as_uint(left0), d = __float_as_uint(left1);
  mid = __byte_perm(c, d, 0x7632);
  lo = __byte_perm(__float_as_uint(left0 - __uint_as_float(c & 0xffff0000u)), __float_as_uint(left1 - __uint_as_float(d & 0xffff0000u)), 0x7632);
}

// A product as the caller described it. whole: 16 bytes of a row of x are one aligned piece.
struct Q4Product {
  const emr_q4* w;
  const void* x;
  int32_t dtype, x_batch;
  int64_t rows, batch_stride, row_stride, col_stride;
  bool whole;
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};
// Whether it is one for the kernel of many rows (emr_q4_many.cu), the bytes that that needs, and its launch. Measured, in us, few and
// many: 4096 x 4096 with 16 rows of bfloat16 7.9 and 10.6, 20 rows 19 and 11, 10 rows of float32 21 and 12; 16384 x 8192 with 16 rows
// 31 and 36, 20 rows 41 and 37, 10 rows of float32 52 and 49; 100 networks of 1364 x 256, where a block's set-up counts for two blocks of
// columns, 24 rows 31 and 38, 32 rows 37 and 39, 16 rows of float32 34 and 43.
inline bool q4_is_many(const Q4Product& a) {
  const int most = a.dtype == EMR_F32 ? 8 : 16;
  return a.rows > (a.w->cols <= 512 ? 2 * most : most);
}
size_t q4_many_room(const Q4Product& a);
emr_status launch_q4_many(const Q4Product& a, void* ws, int dev, int sms, cudaStream_t st);

inline bool q4_ok(const emr_q4* q) {
  return q && q->batch > 0 && q->rows > 0 && q->cols > 0 && q->rows <= kQ8MaxDim && q->cols <= kQ8MaxDim &&
         (q->group == 32 || q->group == 64 || q->group == 128) && q->data && reinterpret_cast<uintptr_t>(q->data) % 16 == 0;
}

}  // namespace emr
