// Device helpers of the block-scaled 8-bit layout (emr_q8 in emr.h), shared by
// the quantising kernels and the matrix product.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

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
  const int b = int((top + 0x1fffffu) >> 23) - 8;  // a fraction above 0x600000 carries into the exponent
  return top == 0 ? 127u : uint32_t(max(b, 1));
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
// Four values times inv as e4m3 codes, rounded to nearest even; v0 is the low byte. NaN
// gives the NaN code; an infinity would saturate (q8_finite_or_nan first).
__device__ __forceinline__ uint32_t q8_pack4(float v0, float v1, float v2, float v3, float inv) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v1 * inv), "f"(v0 * inv));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v3 * inv), "f"(v2 * inv));
  return uint32_t(lo) | (uint32_t(hi) << 16);
}
// Largest magnitude of four values; NaN only where all are.
__device__ __forceinline__ float q8_top4(float4 v) {
  return fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w)));
}
// Scale byte of a block spread over a warp, four values a lane. Blocks with an infinity
// or nothing but NaN in some lane take the second look; there infinities turn into NaN.
__device__ __forceinline__ uint32_t q8_warp_scale(float4& v) {
  uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(q8_top4(v)));
  if (top >= 0x7f800000u) {
    top = __reduce_max_sync(0xffffffffu, max(max(q8_magnitude(v.x), q8_magnitude(v.y)), max(q8_magnitude(v.z), q8_magnitude(v.w))));
    v = make_float4(q8_finite_or_nan(v.x), q8_finite_or_nan(v.y), q8_finite_or_nan(v.z), q8_finite_or_nan(v.w));
  }
  return q8_scale_byte(top);
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
__device__ __forceinline__ void store_scalar(void* p, int dtype, int64_t i, float v) {
  if (dtype == EMR_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == EMR_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
// Four neighbouring elements as they lie in memory, and as floats.
template <typename T>
struct Four {
  uint2 u;
  __device__ __forceinline__ void set(int j, T v) { reinterpret_cast<T*>(&u)[j] = v; }
  __device__ __forceinline__ float4 floats() const {
    const T* e = reinterpret_cast<const T*>(&u);
    return make_float4(float(e[0]), float(e[1]), float(e[2]), float(e[3]));
  }
};
template <>
struct Four<float> {
  float4 u;
  __device__ __forceinline__ void set(int j, float v) { reinterpret_cast<float*>(&u)[j] = v; }
  __device__ __forceinline__ float4 floats() const { return u; }
};
__host__ __device__ inline int dtype_bytes(int dtype) { return dtype == EMR_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == EMR_F32 || dtype == EMR_BF16 || dtype == EMR_F16; }

// Host check of a q8 tensor's description.
inline bool q8_ok(const emr_q8* q) {
  return q && q->batch > 0 && q->rows > 0 && q->cols > 0 && q->rows <= kQ8MaxDim && q->cols <= kQ8MaxDim && q->values &&
         q->scales && reinterpret_cast<uintptr_t>(q->values) % 16 == 0 && reinterpret_cast<uintptr_t>(q->scales) % 16 == 0;
}

// Launches of this library's dense-layer kernels overlap: each begins its set-up while the one
// before it in the stream ends, waits (grid_wait) before it touches memory, and then lets
// the next one begin (grid_go).
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_go() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... P, typename... A>
emr_status launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

// The current device and its number of SMs.
inline bool device_sms(int* dev, int* sms) {
  return cudaGetDevice(dev) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev) == cudaSuccess;
}

// Once for each device and kernel: its dynamic shared memory.
template <typename K>
bool allow_smem(K kernel, int bytes, int dev, std::atomic<uint64_t>& done) {
  if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  if (dev < 64) done.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
  return true;
}

constexpr int kMostSmem = 224 * 1024;  // dynamic, beside at most 3 KB of static arrays

// The product of a few rows of x, quantised within the kernel (emr_q8_few.cu).
struct FewArgs {
  const void* x;
  int32_t x_dtype, x_batch;
  int64_t x_rows, x_batch_stride, x_row_stride, x_col_stride;
  const emr_q8* w;
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype, batch;
};
// Where it takes less time than two launches, or as much: up to 4 MB of weights for at most 8 rows; with one
// or two rows, each of them quantised in every block, up to 8 MB, and 16 where a row is long enough to share out.
inline bool few_fused(int64_t rows, const emr_q8& w) {
  const int64_t row = q8_row_bytes(w.cols), most = rows > 2 ? 4 : row < 1024 ? 8 : 16;
  return rows <= 8 && rows * row <= 8192 && w.batch <= 65535 && double(w.batch) * double(w.rows) * double(row) <= double(most << 20);
}
emr_status launch_few(const FewArgs& a, cudaStream_t st);

}  // namespace emr
