// rope_kernel.cu - rotary positions of a layer's queries and keys.
//
// Column pair i of a row at position t turns by the angle t f_i:
//   y_a = m (x_a cos - x_b sin),  y_b = m (x_a sin + x_b cos)
// with (a, b) = (2i, 2i + 1) or (i, i + R / 2), m the factor of a stretched context, and the
// opposite angle for the inverse, which (the rotation being orthogonal) is the gradient as well.
// Columns R .. D - 1 are copied.
//
// The angle. t f_i reaches 1e5 radians and more, where a product in fp32 is off by 1e-2. The frequency
// is taken as a fraction of a turn in 64-bit fixed point, f_i / 2 pi mod 1: the product with the
// position wraps modulo one turn by itself, exactly, and its upper 32 bits are the reduced angle (off
// by t 2^-53 turns from the fp64 frequency and 2^-26 turns from the conversion to fp32).
//
// Bound by memory: each row is read and written once. A thread holds one 16-byte vector column (two, R / 2
// apart, in the layout of halves) of one token and walks over up to eight heads, so that its sines and cosines serve
// all of them. The first rows and the position are loaded before the frequencies are made ready and waited for (8 x 32 + 32 heads,
// 64 tokens of 64 fp32: 8.7 us without that and with a head a thread, 3.9 so; 4 tokens of 28 + 4 heads 2.9 and 2.4).
// A frequency that is not finite has no turns: the CTA's barrier says whether there is one, and its columns are NaN then (a mark
// among the turns, looked at pair by pair, took 1 % of a prompt's time).
// More threads with fewer loads each are faster than the opposite where the rows come from HBM: 4 x 40 heads, 8191
// tokens of 128 bf16 took 117 us with one head in flight a thread and four CTAs of 256 an SM, 132 with two and three, 165
// with four and two, 253 with eight (2048 tokens of one sequence, which stay in L2: 10.3 and 8.7 with two and three); in
// neighbouring pairs 121 with two heads and four CTAs, 140 with two and three, 162 with four and two; fp32 (32 + 32
// heads, 4096 tokens of 64, halves) 81 with four heads and three CTAs, 94 with four and two or two and three. Walks over
// 16 or 40 heads: 127 and 142 us.
#include <cuda_bf16.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.cuh"
#include "ptx.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;

struct RopeTensor {
  const uint8_t* in;
  uint8_t* out;
  long long in_b, in_h, in_l, out_b, out_h, out_l;   // strides in elements
  int heads;
};

struct RopeParams {
  RopeTensor t[2];         // q, k
  const double* inv_freq;  // [R / 2] radians per position
  const int32_t* pos;      // [B, L] or null: pos0 + l
  int pos0, L, D, R;
  int units;               // a row's work items: one a thread
  int turn_units;          // of them, those that turn (the rest copy columns R .. D - 1)
  int chunk;               // heads a thread walks over
  int chunks0, chunks;     // chunks of q, and of q and k
  long long items;         // B * L * chunks * units
  float mscale;
  int inverse;
};

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

__device__ __forceinline__ int not_finite(double x) { return (__double2hiint(x) & 0x7ff00000) == 0x7ff00000; }

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// T: element; N: elements of a thread's vector (16 bytes, or one element where a size, a stride or
// a pointer does not allow more); kInter: pairs of neighbours (a vector of N >= 2 holds N / 2 pairs).
template <typename T, int N, bool kInter>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kHeadsInFlight = sizeof(T) == 2 ? (kInter ? 2 : 1) : 4;
  extern __shared__ uint64_t turns[];   // [R / 2] fractions of a turn per position, 2^64 = one turn
  const long long item = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
  const bool live = item < p.items;
  int u, c;
  long long rest;                                            // token b * L + l
  if (p.items <= 0x7fffffffLL) {
    const unsigned i = live ? static_cast<unsigned>(item) : 0u, r = i / static_cast<unsigned>(p.units);
    u = static_cast<int>(i - r * static_cast<unsigned>(p.units));
    rest = r / static_cast<unsigned>(p.chunks);
    c = static_cast<int>(r - static_cast<unsigned>(rest) * static_cast<unsigned>(p.chunks));
  } else {
    const long long i = live ? item : 0;
    u = static_cast<int>(i % p.units);
    rest = i / p.units;
    c = static_cast<int>(rest % p.chunks);
    rest /= p.chunks;
  }
  const long long b = rest / p.L;
  const int l = static_cast<int>(rest - b * p.L);
  const bool turn = u < p.turn_units;
  constexpr int kHalf = kInter ? (N >= 2 ? N / 2 : 1) : N;   // pairs of a work item
  constexpr int kVecs = kInter && N >= 2 ? 1 : 2;            // vectors of a turning work item
  // columns of the work item's vectors
  int col0, col1 = 0;
  if (turn) {
    col0 = kInter ? u * (N >= 2 ? N : 2) : u * N;
    col1 = kInter ? col0 + 1 : col0 + p.R / 2;
  } else {
    col0 = p.R + (u - p.turn_units) * N;
  }
  const int which = c >= p.chunks0 ? 1 : 0;
  const RopeTensor& t = p.t[which];
  // heads h0, h0 + step, ...: the chunks' threads, neighbours in a warp, read and write neighbouring heads
  const int step = which ? p.chunks - p.chunks0 : p.chunks0;
  const int h0 = which ? c - p.chunks0 : c;
  const int n = live ? (t.heads - h0 + step - 1) / step : 0;
  const T* in = reinterpret_cast<const T*>(t.in) + b * t.in_b + l * t.in_l;
  T* out = reinterpret_cast<T*>(t.out) + b * t.out_b + l * t.out_l;
  using V = Vec<T, N>;
  V x[kHeadsInFlight][2];
  const auto load = [&](int i0) {
#pragma unroll
    for (int j = 0; j < kHeadsInFlight; ++j) {
      if (i0 + j >= n) break;
      const T* row = in + (h0 + (i0 + j) * step) * t.in_h;
      x[j][0] = *reinterpret_cast<const V*>(row + col0);
      if (kVecs == 2 && turn) x[j][1] = *reinterpret_cast<const V*>(row + col1);
    }
  };
  griddep_wait();
  griddep_launch_dependents();
  // the first rows and the position are on their way while the frequencies are made ready
  int32_t at = static_cast<int32_t>(static_cast<uint32_t>(p.pos0) + l);
  if (p.pos != nullptr && turn) at = p.pos[rest];
  load(0);
  int bad = 0;   // some frequency is not finite: the exponent bits are all set
  for (int i = threadIdx.x; i < p.R / 2; i += kThreads) {
    const double radians = p.inv_freq[i], f = radians * 0.15915494309189535;   // / 2 pi
    turns[i] = __double2ull_rn((f - floor(f)) * 18446744073709551616.0);
    bad |= not_finite(radians);
  }
  bad = __syncthreads_or(bad);
  float cs[kHalf], sn[kHalf];
  if (turn) {
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
      const uint64_t a = static_cast<uint64_t>(static_cast<int64_t>(at)) * turns[u * kHalf + i];
      // the nearest of 2^-32 turns, in units of pi: [-1, 1]
      const float x = static_cast<float>(static_cast<int32_t>((a + 0x80000000ull) >> 32)) * 4.656612873077393e-10f;
      float s, co;
      sincospif(x, &s, &co);
      cs[i] = co * p.mscale;
      sn[i] = (p.inverse ? -s : s) * p.mscale;
    }
    if (bad) {
#pragma unroll
      for (int i = 0; i < kHalf; ++i)
        if (not_finite(p.inv_freq[u * kHalf + i])) cs[i] = sn[i] = __uint_as_float(0x7fc00000u);
    }
  }
  for (int i0 = 0; i0 < n; i0 += kHeadsInFlight) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int j = 0; j < kHeadsInFlight; ++j) {
      if (i0 + j >= n) break;
      T* row = out + (h0 + (i0 + j) * step) * t.out_h;
      if (turn) {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          T& xa = kVecs == 1 ? x[j][0].v[(2 * i) % N] : x[j][0].v[i % N];
          T& xb = kVecs == 1 ? x[j][0].v[(2 * i + 1) % N] : x[j][1].v[i % N];
          const float a = to_f(xa), d = to_f(xb);
          xa = from_f<T>(a * cs[i] - d * sn[i]);
          xb = from_f<T>(a * sn[i] + d * cs[i]);
        }
      }
      *reinterpret_cast<V*>(row + col0) = x[j][0];
      if (kVecs == 2 && turn) *reinterpret_cast<V*>(row + col1) = x[j][1];
    }
  }
}

// Whether every row of the tensor starts on a vector of n elements of e bytes.
bool vectors_fit(const RopeTensor& t, int n, int e) {
  if (t.heads == 0) return true;
  const auto fits = [&](const void* p) { return reinterpret_cast<uintptr_t>(p) % (static_cast<size_t>(n) * e) == 0; };
  return fits(t.in) && fits(t.out) && t.in_b % n == 0 && t.in_h % n == 0 && t.in_l % n == 0 && t.out_b % n == 0 &&
         t.out_h % n == 0 && t.out_l % n == 0;
}

}  // namespace

int launch_rope(const RopeArgs& a, cudaStream_t stream) {
  RopeParams p{};
  for (int i = 0; i < 2; ++i) {
    const int64_t* s = a.strides + 3 * i;
    p.t[i] = RopeTensor{static_cast<const uint8_t*>(i ? a.k : a.q), static_cast<uint8_t*>(i ? a.k_out : a.q_out),
                        s[0], s[1], s[2], s[6], s[7], s[8], i ? a.Hkv : a.Hq};
  }
  p.inv_freq = a.inv_freq;
  p.pos = a.pos;
  p.pos0 = a.pos0;
  p.L = a.L;
  p.D = a.D;
  p.R = a.R;
  p.mscale = a.mscale;
  p.inverse = a.inverse;
  const int e = a.elem_bytes;
  int n = 16 / e;
  const bool wide = vectors_fit(p.t[0], n, e) && vectors_fit(p.t[1], n, e) && a.D % n == 0 &&
                    (a.interleaved ? a.R % n == 0 : (a.R / 2) % n == 0);
  if (!wide) n = 1;
  const int per_unit = a.interleaved ? (n >= 2 ? n / 2 : 1) : n;   // pairs of a work item
  p.turn_units = a.R / 2 / per_unit;
  p.units = p.turn_units + (a.D - a.R) / n;
  // Heads a thread walks over: all work items of a small call are spread over the GPU (one head each), a
  // large call's threads share their sines and cosines between eight heads. In between two CTAs an SM are enough: 8 x
  // 64 heads, 64 tokens of 128 fp32 take 6.0 us so and 11.9 with eight (256 threads more or less an SM: 5.2, 6.5).
  const long long tokens = static_cast<long long>(a.B) * a.L;
  const long long all = tokens * p.units * (a.Hq + a.Hkv);
  p.chunk = static_cast<int>(std::min<long long>(8, std::max<long long>(1, all / (152 * 512))));
  p.chunks0 = (a.Hq + p.chunk - 1) / p.chunk;
  p.chunks = p.chunks0 + (a.Hkv + p.chunk - 1) / p.chunk;
  p.items = tokens * p.chunks * p.units;
  const long long grid = (p.items + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffLL) return -2;
  if (grid == 0) return 0;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads),
                                            static_cast<size_t>(a.R / 2) * 8, stream, attr);
  using bf16 = __nv_bfloat16;
  cudaError_t r;
  if (e == 2)
    r = wide ? (a.interleaved ? cudaLaunchKernelEx(&cfg, rope_kernel<bf16, 8, true>, p)
                              : cudaLaunchKernelEx(&cfg, rope_kernel<bf16, 8, false>, p))
             : (a.interleaved ? cudaLaunchKernelEx(&cfg, rope_kernel<bf16, 1, true>, p)
                              : cudaLaunchKernelEx(&cfg, rope_kernel<bf16, 1, false>, p));
  else
    r = wide ? (a.interleaved ? cudaLaunchKernelEx(&cfg, rope_kernel<float, 4, true>, p)
                              : cudaLaunchKernelEx(&cfg, rope_kernel<float, 4, false>, p))
             : (a.interleaved ? cudaLaunchKernelEx(&cfg, rope_kernel<float, 1, true>, p)
                              : cudaLaunchKernelEx(&cfg, rope_kernel<float, 1, false>, p));
  return r == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
