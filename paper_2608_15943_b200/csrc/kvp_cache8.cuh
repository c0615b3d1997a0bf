// e4m3 numbers on the device: conversions of two or four at a time.
#pragma once
#include <cuda_fp16.h>

#include "kvp_cache8.h"
#include "kvp_sm100.cuh"

namespace kvp {

// two e4m3 numbers (low byte first) as two f16, exactly
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
  return r;
}
// to the nearest e4m3, ties to even; NaN stays NaN
__device__ __forceinline__ uint32_t f32x4_to_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return uint32_t(lo) | uint32_t(hi) << 16;
}
__device__ __forceinline__ float2 f16x2_to_f32(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
// four e4m3 numbers times a power of two, rounded again
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t v, float factor) {
  const float2 a = f16x2_to_f32(e4m3x2_to_f16x2(uint16_t(v))), b = f16x2_to_f32(e4m3x2_to_f16x2(uint16_t(v >> 16)));
  return f32x4_to_e4m3(a.x * factor, a.y * factor, b.x * factor, b.y * factor);
}

}  // namespace kvp
