// What the kernels on rows of scores share: 16 bytes of scores, and the order of scores as integers.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace emr {

// Order-preserving integer of a score that is not masked; masked ones give 0.
__device__ __forceinline__ uint32_t order_key(float s) {
  if (!(s > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(s + 0.f);  // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_score(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// 16 bytes of scores.
template <typename T>
struct Group {
  static constexpr int kSize = 16 / int(sizeof(T));
  uint4 u;
  __device__ __forceinline__ void set(int j, T v) { reinterpret_cast<T*>(&u)[j] = v; }
  __device__ __forceinline__ void mask(int j) { set(j, T(-INFINITY)); }
  __device__ __forceinline__ float get(int j) const { return float(reinterpret_cast<const T*>(&u)[j]); }
};

}  // namespace emr
