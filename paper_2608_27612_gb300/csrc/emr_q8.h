// Device helpers of the block-scaled 8-bit layout (emr_q8 in emr.h), shared by
// the quantising kernels and the matrix product.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/emr.h"

namespace emr {

constexpr int kQ8Block = 128;  // values that share a scale, and rows of a scale tile
constexpr int64_t kQ8MaxDim = (int64_t(1) << 31) - 256;

__host__ __device__ inline int64_t q8_blocks(int64_t n) { return (n + kQ8Block - 1) / kQ8Block; }
__host__ __device__ inline int64_t q8_row_bytes(int64_t cols) { return q8_blocks(cols) * kQ8Block; }
// 512-byte scale tiles of one row tile: four blocks of 128 columns each.
__host__ __device__ inline int64_t q8_scale_chunks(int64_t cols) { return (q8_blocks(cols) + 3) / 4; }
__host__ __device__ inline int64_t q8_scale_batch(int64_t rows, int64_t cols) {
  return q8_blocks(rows) * q8_scale_chunks(cols) * 512;
}
// Byte of the scale of row r, column block kb: tiles of 128 rows x 4 blocks in
// the order in which the tensor core's scale memory takes them: row % 32 picks
// 16 bytes, row / 32 a word of those, the block a byte of the word.
__host__ __device__ inline int64_t q8_scale_at(int64_t chunks, int64_t r, int64_t kb) {
  return ((r >> 7) * chunks + (kb >> 2)) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (kb & 3);
}

// Scale byte of a block whose largest finite magnitude has the bits `top`: 127 + e
// for the least e with top <= 448 * 2^e (448 = 1.75 * 2^8 is e4m3's largest value);
// e is at least -126, and 0 for a block of zeros.
__device__ __forceinline__ uint32_t q8_scale_byte(uint32_t top) {
  if (top == 0) return 127u;
  const int b = int(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return uint32_t(b < 1 ? 1 : b);
}
__device__ __forceinline__ float q8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float q8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Magnitude bits of v for the block's maximum; infinities and NaN do not count
// (they become the NaN code and leave the block's other values as they are).
__device__ __forceinline__ uint32_t q8_magnitude(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
__device__ __forceinline__ float q8_finite_or_nan(float v) {
  return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : v;
}
// Four values times inv as e4m3 codes, rounded to nearest even; v0 is the low byte.
__device__ __forceinline__ uint32_t q8_pack4(float v0, float v1, float v2, float v3, float inv) {
  uint16_t lo, hi;
  const float a = q8_finite_or_nan(v0) * inv, b = q8_finite_or_nan(v1) * inv;
  const float c = q8_finite_or_nan(v2) * inv, d = q8_finite_or_nan(v3) * inv;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return uint32_t(lo) | (uint32_t(hi) << 16);
}
// The values that four codes stand for, before the scale.
__device__ __forceinline__ float4 q8_unpack4(uint32_t p) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(uint16_t(p)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(uint16_t(p >> 16)));
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return make_float4(a.x, a.y, b.x, b.y);
}

// Element i of an array of the given emr_dtype.
__device__ __forceinline__ float load_scalar(const void* p, int dtype, int64_t i) {
  if (dtype == EMR_F32) return static_cast<const float*>(p)[i];
  if (dtype == EMR_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_scalar(void* p, int dtype, int64_t i, float v) {
  if (dtype == EMR_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == EMR_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
// Elements i .. i + 3, aligned to their four-element size.
__device__ __forceinline__ float4 load_four(const void* p, int dtype, int64_t i) {
  if (dtype == EMR_F32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
  const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
  float2 a, b;
  if (dtype == EMR_BF16) {
    a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
    b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  } else {
    a = __half22float2(*reinterpret_cast<const __half2*>(&u.x));
    b = __half22float2(*reinterpret_cast<const __half2*>(&u.y));
  }
  return make_float4(a.x, a.y, b.x, b.y);
}
__host__ __device__ inline int dtype_bytes(int dtype) { return dtype == EMR_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == EMR_F32 || dtype == EMR_BF16 || dtype == EMR_F16; }

// Host check of a q8 tensor's description.
inline bool q8_ok(const emr_q8* q) {
  return q && q->batch > 0 && q->rows > 0 && q->cols > 0 && q->rows <= kQ8MaxDim && q->cols <= kQ8MaxDim && q->values &&
         q->scales && reinterpret_cast<uintptr_t>(q->values) % 16 == 0 && reinterpret_cast<uintptr_t>(q->scales) % 16 == 0;
}

}  // namespace emr
