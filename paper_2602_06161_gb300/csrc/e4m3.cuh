// e4m3.cuh - rows of the 8-bit memory: e4m3 codes with one e8m0 exponent byte a row.
//
// A row's values are code * 2^(x - 127), x its byte (255: the row reads as NaN). A power of two scales
// without rounding, so every value is exact in bf16 and in fp32, and quantising loses what e4m3's three
// mantissa bits lose and nothing else: |error| <= 2^-4 of the value, or 2^(x - 127 - 10) where that
// is more.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace cover {

constexpr int kExpNan = 255;    // a row with an element that is not finite
constexpr int kExpZero = 127;   // a row of zeros
// The bytes written are held to 2^-110 .. 2^119: 448 * 2^119 is the largest of them that bf16 holds, and at
// 2^-110 the smallest code, 2^-9, is still a normal number.
constexpr int kExpMin = 17, kExpMax = 246;

// The smallest byte x with amax <= 448 * 2^(x - 127) (448 = 1.75 * 2^8), from the bits of amax >= 0.
__device__ __forceinline__ int e4m3_row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int biased = static_cast<int>(u >> 23);
  if (biased == 255) return kExpNan;
  if (u == 0) return kExpZero;
  const int x = biased - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(x, kExpMin), kExpMax);
}

// 2^(127 - x) for a byte that e4m3_row_exponent wrote; 0 for a NaN row, whose codes are zeros.
__device__ __forceinline__ float e4m3_inverse_scale(int x) {
  return x == kExpNan ? 0.0f : __uint_as_float(static_cast<uint32_t>(254 - x) << 23);
}

// 2^(x - 127) of any byte, NaN for 255.
__device__ __forceinline__ float e4m3_scale(int x) {
  return __uint_as_float(x == 0 ? 0x00400000u : x == kExpNan ? 0x7fc00000u : static_cast<uint32_t>(x) << 23);
}

// Two codes of the low and the high half: nearest, ties to even, saturating at 448.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// The values of two codes (exact in fp16).
__device__ __forceinline__ float2 e4m3x2_values(uint32_t codes) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xffffu), __NV_E4M3);
  return __half22float2(__half2(h));
}

}  // namespace cover
