// fp8.cuh -- e4m3 values with a power-of-two scale per KV page and head.
#pragma once

#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace wisp {

// Exponents of the scales that the library writes: far inside fp32, so that scales, their reciprocals and
// scaled values never leave it.
constexpr int kScaleExpMin = -96, kScaleExpMax = 120;

// Sums of scaled values in fp32: from the first scale above kLargeScale on they are taken times kSumDown (and kSumDownLog2 is added to
// the maximum that goes with them), so that up to 2^20 of the largest values stay finite.
constexpr float kLargeScale = 0x1p64f, kSumDown = 0x1p-20f, kSumDownLog2 = 20.0f;

// two values -> two e4m3 codes (a in the low byte): round to nearest even, past +-448 (and +-inf) to +-448,
// NaN to NaN
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// two e4m3 codes (in the low 16 bits) -> two halves, exactly
__device__ __forceinline__ uint32_t e4m3x2_to_h2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
  return r;
}
__device__ __forceinline__ float2 h2_to_f2(uint32_t h2) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&h2));
}

// The least e with amax <= 448 * 2^e, within the exponents above (0 for amax = 0): 448 = 1.75 * 2^8, so e is the
// exponent of amax less 8, and one more where its significand is above 1.75.  amax is finite.
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  if (b == 0) return 0;
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);  // (subnormal: far below the least)
  return min(max(e, kScaleExpMin), kScaleExpMax);
}
__device__ __forceinline__ float exp2i(int e) { return __int_as_float((e + 127) << 23); }  // e a normal exponent

}  // namespace wisp
