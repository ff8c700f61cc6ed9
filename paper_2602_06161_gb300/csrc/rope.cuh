// rope.cuh - angles of rotary positions (rope_kernel.cu says how they are reduced), and the row vectors of the kernels that turn
// rows by them.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace cover {

// A frequency in radians per position as a fraction of a turn, 2^64 = one turn.
__device__ __forceinline__ uint64_t rope_turns(double radians) {
  const double f = radians * 0.15915494309189535;   // / 2 pi
  return __double2ull_rn((f - floor(f)) * 18446744073709551616.0);
}

__device__ __forceinline__ int not_finite(double x) { return (__double2hiint(x) & 0x7ff00000) == 0x7ff00000; }

// Sine and cosine of position `at` times a frequency.
__device__ __forceinline__ void rope_sincos(int64_t at, uint64_t turns, float* s, float* c) {
  const uint64_t a = static_cast<uint64_t>(at) * turns;
  // the nearest of 2^-32 turns, in units of pi: [-1, 1]
  const float x = static_cast<float>(static_cast<int32_t>((a + 0x80000000ull) >> 32)) * 4.656612873077393e-10f;
  sincospif(x, s, c);
}

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f(float x) {
  return x;
}
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 x) {
  return __bfloat162float(x);
}
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f(float x) {
  return x;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float x) {
  return __float2bfloat16_rn(x);
}

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

}  // namespace cover
