// The six activations and their slopes on a thread's registers, for the dense layers.
#pragma once

#include <cuda_runtime.h>

#include "../../include/emr.h"

namespace emr {

// The transcendental parts run on the special function unit. sigmoid and tanh are taken
// from t = e^-|z| or e^-2|z| and r = 1 / (1 + t): every form below is a product of
// positive terms, so the slopes keep their relative precision where the functions
// saturate (1 - y^2 would lose it).

__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_log2(float x) {
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2E = 0x1.715476p+0f;

// Element i of sin and cos where the argument is large; i is not known at compile time, so the
// element is picked by comparison instead of by an address.
template <int kN, bool kSlope>
__device__ __forceinline__ void sin_far(float (&z)[kN], float (&d)[kN], int i) {
  float v = 0.f, c;
#pragma unroll
  for (int j = 0; j < kN; j++) v = j == i ? z[j] : v;
  sincosf(v, &v, &c);
#pragma unroll
  for (int j = 0; j < kN; j++) {
    z[j] = j == i ? v : z[j];
    if (kSlope) d[j] = j == i ? c : d[j];
  }
}

template <int kN, bool kSlope>
__device__ __forceinline__ void activate(int act, float (&z)[kN], float (&d)[kN]) {
  switch (act) {
    case EMR_ACT_SIGMOID:
#pragma unroll
      for (int i = 0; i < kN; i++) {
        const float t = fast_exp2(fabsf(z[i]) * -kLog2E), r = fast_rcp(1.f + t);
        if (kSlope) d[i] = t * r * r;
        z[i] = z[i] >= 0.f ? r : t * r;
      }
      break;
    case EMR_ACT_TANH:
#pragma unroll
      for (int i = 0; i < kN; i++) {
        const float t = fast_exp2(fabsf(z[i]) * (-2.f * kLog2E)), r = fast_rcp(1.f + t);
        if (kSlope) d[i] = (4.f * t) * (r * r);
        // below 1/25 two terms of the series; the next one is 2 z^4 / 15 (relative 4e-7)
        const float series = z[i] * fmaf(z[i] * z[i], -1.f / 3.f, 1.f);
        z[i] = fabsf(z[i]) < 0.04f ? series : copysignf((1.f - t) * r, z[i]);
      }
      break;
    case EMR_ACT_GAUSS:
#pragma unroll
      for (int i = 0; i < kN; i++) {
        const float y = fast_exp2(z[i] * (z[i] * -kLog2E));
        if (kSlope) d[i] = y == 0.f ? 0.f : -2.f * z[i] * y;  // an infinite z has slope 0
        z[i] = y;
      }
      break;
    case EMR_ACT_SIN: {
      // reduced by 2 pi in two parts (fp32 value and remainder) and taken by the special
      // function unit, good to 1e-6 up to 8192; beyond that, and for infinities, by sincosf. NaN is
      // passed over by the maximum and stays NaN either way.
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < kN; i++) most = fmaxf(most, fabsf(z[i]));
      if (most < 8192.f) {
#pragma unroll
        for (int i = 0; i < kN; i++) {
          const float k = fmaf(z[i], 0x1.45f306p-3f, 0x1.8p+23f) - 0x1.8p+23f;  // nearest whole number of periods
          const float r = fmaf(-k, -0x1.777a5cp-23f, fmaf(-k, 0x1.921fb6p+2f, z[i]));
          if (kSlope) d[i] = __cosf(r);
          z[i] = __sinf(r);
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < kN; i++) sin_far<kN, kSlope>(z, d, i);
      }
      break;
    }
    case EMR_ACT_ABS:
#pragma unroll
      for (int i = 0; i < kN; i++) {
        if (kSlope) d[i] = z[i] > 0.f ? 1.f : z[i] < 0.f ? -1.f : z[i];  // 0 at 0, NaN at NaN
        z[i] = fabsf(z[i]);
      }
      break;
    default:
      if (kSlope) {
#pragma unroll
        for (int i = 0; i < kN; i++) d[i] = 1.f;
      }
  }
}

}  // namespace emr
