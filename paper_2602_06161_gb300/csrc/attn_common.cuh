// attn_common.cuh - device helpers that the window attention kernels share (attn_prefix8.cu, attn_paged.cu): waits of a warp,
// capped scores, and 16-column accesses to tensor memory.
#pragma once

#include <math.h>
#include <stdint.h>

#include "ptx.cuh"

namespace cover {

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  const bool ok = mbar_wait(bar, parity, abort);
  return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// tanh(x) / x = T0 + T1 z + T2 z^2 + T3 z^3 with z = x^2 for |x| <= 0.4: the polynomial through the function at 2000
// Chebyshev nodes of z in [0, 0.16] by least squares, off by at most 1e-7 of it (2e-7 in fp32). Scores are seldom above
// 0.4 of their cap, and then two special-function operations an element are saved.
constexpr float kTanhRange = 0.4f;
constexpr float kMaxCap = 1.1529215e18f;   // 2^60: larger caps count as this one; its reciprocal times the rows' scales is a normal number
// 2^-30: smaller caps count as this one, whose scores change no weight in fp32 (its reciprocal is a number, 0 times infinity none)
constexpr float kMinCap = 9.3132257e-10f;
constexpr float kTanh0 = 0.999999903f, kTanh1 = -0.333313733f, kTanh2 = 0.132711566f, kTanh3 = -0.0475610772f;

// Shared memory by its 32-bit address.
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// A capped score in log2 units, c tanh(s / c) log2(e) = C (1 - 2 / (1 + 2^y)), C = c log2(e), y = 2 log2(e) s / c
// (y = s cap_in); the infinite and the vanishing exponential give the caps themselves. That is off by 2^-23 of the cap, so
// for |s / c| <= 0.4 it is C x P(x^2) instead, off by 2e-7 of the score: a cap far above the scores changes nothing.
__device__ __forceinline__ float capped(float s, float cap_in, float cap_log2) {
  constexpr float kX = 0.34657359f, kX2 = kX * kX;   // x = y ln(2) / 2
  constexpr float a0 = kTanh0 * kX, a1 = kTanh1 * kX * kX2, a2 = kTanh2 * kX * kX2 * kX2, a3 = kTanh3 * kX * kX2 * kX2 * kX2;
  const float y = s * cap_in, z = y * y;
  const float far = fmaf(-2.0f * cap_log2, rcp_approx(1.0f + ex2_approx(y)), cap_log2);
  const float near = cap_log2 * y * fmaf(z, fmaf(z, fmaf(z, a3, a2), a1), a0);
  return fabsf(y) <= kTanhRange / kX ? near : far;
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// Completes the warp's loads; the registers pass through so that none is used before.
__device__ __forceinline__ void tmem_ld_wait16(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ float max32(const float (&s)[32]) {
  float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
  for (int c = 4; c + 8 <= 32; c += 8)
#pragma unroll
    for (int e = 0; e < 4; ++e) mx[e] = fmax3(mx[e], s[c + 2 * e], s[c + 2 * e + 1]);
  mx[0] = fmax3(mx[0], s[28], s[29]);
  mx[1] = fmax3(mx[1], s[30], s[31]);
  return fmax3(mx[0], mx[1], fmaxf(mx[2], mx[3]));
}

// fp32 numbers as integers of the same order (no NaN), and back.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

}  // namespace cover
