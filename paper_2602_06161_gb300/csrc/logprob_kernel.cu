// logprob_kernel.cu - log probabilities of given tokens, with entropy and the best alternatives, and their gradient.
//
// Per row x of V logits, with m a reference, S = sum_j e^(x_j - m), W = sum_j (x_j - m) e^(x_j - m):
//   lse = m + ln S,  log p(y) = (x_y - m) - ln S,  H = -sum_j p_j ln p_j = ln S - W / S
// (H relative to the reference: no difference of numbers as large as the logits). A logit of -inf has p = 0
// and adds nothing. The K best tokens are ordered by (logit descending, index ascending).
//
// Gradient: with a = g_lse - g_y - sum_k g_k - g_H H,
//   d_j = p_j (a - g_H ln p_j) + [j = y] g_y + sum_k [j = idx_k] g_k,   p_j = e^(x_j - lse).
//
// Rows are taken as 16-byte vectors from the one that holds their first element on: rows of any V start at
// any element, and the vectors at a row's two ends are read element by element.
//
// The sums. A thread's reference m is a logit; t_j = x_j log2(e) - c with c = fl(m log2(e)) is one fused operation, and what c is off by
// is known, m log2(e) - c, and taken out of the thread's sums at its end. The reference follows a thread's maximum when that is above it
// by more than kSlack. Logits far below it, -inf among them, are raised to where their weight still is 0 (0 * -inf would be NaN).
// References beyond 2^20, where that correction is no small one, and infinities are left to a second, careful walk.
//
// The K best. Thread t of a CTA keeps the best of its vectors (every 256th) as (largest element, vector). The K-th best of the
// threads' pairs is behind or among the K best vectors, so every one of the K best elements lies in a vector whose pair
// is not behind it, and those are among the K threads in front: their vectors are read again (they are in L2), and the elements that
// are not behind the bound are ranked by counting. What passes the bound is little more than K, whatever ties there are (a row
// of equal logits: the first K vectors). A row whose K best crowd in a few threads may pass more than kMaxFound: then
// the K best are taken one after the other, a walk over the row each.
//
// Few rows are split over the CTAs of a cluster, whose sums and K best its first CTA puts together.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "cluster.cuh"
#include "kernels.cuh"
#include "ptx.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxFound = 1024;        // elements ranked at once
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -1000.0f;     // log2 units: 2^kFloor is 0, and 0 * kFloor too (0 * -inf is not)
constexpr float kSlack = 6.0f;         // the reference follows maxima that are above it by more
constexpr int kMaxParts = 8;           // of a row: CTAs of a cluster

// Elements of a 16-byte vector in fp32.
template <typename T>
struct Vec16;
template <>
struct Vec16<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
  // 2 elements at once: the larger of each (NaN stays), and the largest element of the vector (NaN is passed over)
  static __device__ __forceinline__ uint32_t raised(uint32_t x, uint32_t floor) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(floor));
    return d;
  }
  static __device__ __forceinline__ uint4 raise(const uint4& r, uint32_t floor) {
    return make_uint4(raised(r.x, floor), raised(r.y, floor), raised(r.z, floor), raised(r.w, floor));
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t x, uint32_t y) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y));
    return d;
  }
  static __device__ __forceinline__ float top(const uint4& r) {
    const uint32_t t = larger(larger(r.x, r.y), larger(r.z, r.w));
    return fmaxf(__uint_as_float(t << 16), __uint_as_float(t & 0xffff0000u));
  }
  // x rounded towards -inf, in both halves
  static __device__ __forceinline__ uint32_t floor_of(float x) {
    const uint32_t u = __float_as_uint(x), h = (x < 0.0f ? u + 0xffffu : u) >> 16;
    return h | (h << 16);
  }
  static __device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Vec16<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ uint32_t raised(uint32_t x, uint32_t floor) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(__uint_as_float(x)), "f"(__uint_as_float(floor)));
    return __float_as_uint(d);
  }
  static __device__ __forceinline__ uint4 raise(const uint4& r, uint32_t floor) {
    return make_uint4(raised(r.x, floor), raised(r.y, floor), raised(r.z, floor), raised(r.w, floor));
  }
  static __device__ __forceinline__ float top(const uint4& r) {
    return fmax3(__uint_as_float(r.x), __uint_as_float(r.y), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
  }
  static __device__ __forceinline__ uint32_t floor_of(float x) { return __float_as_uint(x); }
  static __device__ __forceinline__ float value(float v) { return v; }
  static __device__ __forceinline__ float from(float v) { return v; }
};

// The larger of two numbers, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// fp32 numbers as unsigned integers of the same order, above 0 (NaN lies at the ends), and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // -0 counts as 0
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __uint_as_float(u ^ ((u & 0x80000000u) != 0 ? 0x80000000u : 0xffffffffu));
}
// (value, index) as one number: a larger value is in front, of equal ones the lower index. 0: none.
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t i) {
  return (static_cast<unsigned long long>(ordered(x)) << 32) | (0xffffffffu - i);
}
__device__ __forceinline__ uint32_t index_of(unsigned long long key) { return 0xffffffffu - static_cast<uint32_t>(key); }

// A row of V elements as vectors: element j is element j + skip of the vectors from `base` on.
template <typename T>
struct Row {
  const uint4* base;
  int skip, V, n_vecs;
  int whole0, whole1;   // vectors that hold elements of this row alone
  __device__ __forceinline__ Row(const T* logits, long long row, int V) : V(V) {
    constexpr int N = Vec16<T>::kN;
    const T* first = logits + row * V;
    skip = static_cast<int>((reinterpret_cast<uintptr_t>(first) & 15) / sizeof(T));
    base = reinterpret_cast<const uint4*>(first - skip);
    n_vecs = static_cast<int>((static_cast<long long>(V) + skip + N - 1) / N);
    whole0 = skip > 0 ? 1 : 0;
    whole1 = static_cast<int>((static_cast<long long>(V) + skip) / N);
  }
  __device__ __forceinline__ bool whole(int i) const { return i >= whole0 && i < whole1; }
  // whether element e of vector i is in the row
  __device__ __forceinline__ bool has(int i, int e) const {
    const long long j = static_cast<long long>(i) * Vec16<T>::kN + e - skip;
    return j >= 0 && j < V;
  }
  // a vector at the row's ends, -inf in the places of other rows
  __device__ __forceinline__ uint4 load_end(int i) const {
    constexpr int N = Vec16<T>::kN;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e)
      x[e] = has(i, e) ? Vec16<T>::value(reinterpret_cast<const T*>(base)[static_cast<long long>(i) * N + e]) : -INFINITY;
    return Vec16<T>::pack(x);
  }
  __device__ __forceinline__ uint4 load(int i) const { return whole(i) ? __ldg(base + i) : load_end(i); }
};

// Sums of exponentials relative to the logit m: s of 2^t, w of t 2^t, t = (x - m) log2(e). m = -inf: none yet.
struct Sums {
  float m, s, w;
  __device__ __forceinline__ void move_to(float to) {
    const float d = fmaxf((m - to) * kLog2e, kFloor), f = ex2_approx(d);
    w = fmaf(s, d, w) * f;
    s *= f;
    m = to;
  }
};
__device__ __forceinline__ Sums merge(Sums a, Sums b) {
  const float to = fmaxf(a.m, b.m);
  a.move_to(to);
  b.move_to(to);
  return Sums{to, a.s + b.s, a.w + b.w};
}

struct FwdParams {
  const void* logits;
  const int32_t* tok;
  float* logp;
  float* entropy;
  float* lse;
  int32_t* top_idx;
  float* top_logp;
  int V, topk, parts;
};

// A thread's sums over vectors i, i + kThreads, .. below end, for logits of any size.
template <typename T>
__device__ __noinline__ Sums careful_sums(const Row<T>& row, int i, int end) {
  constexpr int N = Vec16<T>::kN;
  Sums a{-INFINITY, 0.0f, 0.0f};
  for (int k = i; k < end; k += kThreads) a.m = fmaxf(a.m, Vec16<T>::top(row.load(k)));
  for (int k = i; k < end; k += kThreads) {
    float x[N];
    Vec16<T>::unpack(row.load(k), x);
    for (int e = 0; e < N; ++e) {
      if (x[e] == -INFINITY) continue;
      const float t = max_nan((x[e] - a.m) * kLog2e, kFloor), f = ex2_approx(t);
      a.s += f;
      a.w = fmaf(f, t, a.w);
    }
  }
  return a;
}

template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads, 4) logprob_fwd_kernel(const __grid_constant__ FwdParams p) {
  using V16 = Vec16<T>;
  constexpr int N = V16::kN, kInFlight = 4;
  __shared__ Sums s_sums[kWarps], s_part;
  __shared__ unsigned long long s_groups[kTop ? kThreads : 1], s_found[kTop ? kMaxFound : 1], s_best[kTop ? kMaxTopLogprob : 1];
  __shared__ unsigned long long s_bound;
  __shared__ int s_who[kTop ? kMaxTopLogprob : 1], s_n_found;
  __shared__ float2 s_row;   // m and ln s of the whole row
  griddep_wait();
  griddep_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = p.parts > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const long long r = blockIdx.x / p.parts;
  const Row<T> row(static_cast<const T*>(p.logits), r, p.V);
  const int each = (row.n_vecs + p.parts - 1) / p.parts;
  const int v0 = min(part * each, row.n_vecs), v1 = min(v0 + each, row.n_vecs);
  float x_tok = 0.0f;
  bool has_tok = false;
  if (tid == 0 && part == 0 && p.tok != nullptr) {
    const int y = __ldg(p.tok + r);
    has_tok = y >= 0 && y < p.V;
    if (has_tok) x_tok = V16::value(static_cast<const T*>(p.logits)[r * p.V + y]);
  }
  if constexpr (kTop) {
    if (tid == 0) s_n_found = 0;
    if (tid < kMaxTopLogprob) s_best[tid] = 0;   // (NaN may leave places empty)
  }

  // ---------------- sums, and each thread's best vector ----------------
  Sums a{-INFINITY, 0.0f, 0.0f};
  bool careful = false;
  {
    constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // -inf
    float c = -INFINITY;
    uint32_t floor = kNone;
    uint64_t s2[2] = {0, 0}, w2[2] = {0, 0};
    float best = 0.0f;
    int best_vec = -1;
    for (int i0 = v0 + tid; i0 < v1; i0 += kThreads * kInFlight) {
      uint4 raw[kInFlight];
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) {
        const int i = i0 + k * kThreads;
        raw[k] = i < v1 ? row.load(i) : make_uint4(kNone, kNone, kNone, kNone);
      }
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) {
        const float t = V16::top(raw[k]);
        const int i = i0 + k * kThreads;
        if (kTop && (t > best || best_vec < 0) && i < v1) best = t, best_vec = i;
        top = fmaxf(top, t);
      }
      if (top > a.m + kSlack) {
        careful |= fabsf(top) > 1048576.0f;
        const float to = top * kLog2e, d = fmaxf(c - to, kFloor), f = ex2_approx(d);
        const uint64_t f2 = f2_pack(f, f), d2 = f2_pack(d, d);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          w2[e] = f2_mul(f2_fma(s2[e], d2, w2[e]), f2);
          s2[e] = f2_mul(s2[e], f2);
        }
        a.m = top;
        c = to;
        floor = V16::floor_of(top - 800.0f);
      }
      if (a.m == -INFINITY) {   // nothing but -inf, or NaN, so far
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
          float x[N];
          V16::unpack(raw[k], x);
#pragma unroll
          for (int e = 0; e < N; ++e) careful |= x[e] != x[e];
        }
        continue;
      }
      const uint64_t l2 = f2_pack(kLog2e, kLog2e), c2 = f2_pack(-c, -c);
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) {
        float x[N];
        V16::unpack(V16::raise(raw[k], floor), x);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const uint64_t t2 = f2_fma(f2_pack(x[e], x[e + 1]), l2, c2);
          float t0, t1;
          f2_unpack(t2, t0, t1);
          const uint64_t e2 = f2_pack(ex2_approx(t0), ex2_approx(t1));
          s2[(e >> 1) & 1] = f2_add(s2[(e >> 1) & 1], e2);
          w2[(e >> 1) & 1] = f2_fma(e2, t2, w2[(e >> 1) & 1]);
        }
      }
    }
    if (careful) {
      a = careful_sums(row, v0 + tid, v1);
    } else if (a.m != -INFINITY) {
      float x[4];
      f2_unpack(f2_add(s2[0], s2[1]), x[0], x[1]);
      f2_unpack(f2_add(w2[0], w2[1]), x[2], x[3]);
      const float off = fmaf(a.m, kLog2e, -c), f = ex2_approx(-off);
      a.s = (x[0] + x[1]) * f;
      a.w = fmaf(-off, x[0] + x[1], x[2] + x[3]) * f;
    }
    if constexpr (kTop) s_groups[tid] = best_vec >= 0 ? key_of(best, static_cast<uint32_t>(best_vec)) : 0ull;
  }
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1)
    a = merge(a, Sums{__shfl_xor_sync(0xffffffffu, a.m, d), __shfl_xor_sync(0xffffffffu, a.s, d), __shfl_xor_sync(0xffffffffu, a.w, d)});
  if (lane == 0) s_sums[warp] = a;
  __syncthreads();
  if (tid == 0) {
    Sums t = s_sums[0];
    for (int i = 1; i < kWarps; ++i) t = merge(t, s_sums[i]);
    s_part = t;
  }
  const int K = kTop ? min(p.topk, p.V) : 0;
  if constexpr (kTop) {
    // ---------------- the part's K best ----------------
    if (warp == 0) {
      // the K best pairs of the 256, a lane's eight in order first
      constexpr int kEach = kThreads / 32;
      unsigned long long mine[kEach];
      int who[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        mine[i] = s_groups[32 * i + lane];
        who[i] = 32 * i + lane;
      }
#pragma unroll
      for (int i = 1; i < kEach; ++i)
#pragma unroll
        for (int j = i; j > 0; --j)
          if (mine[j] > mine[j - 1]) {
            const unsigned long long x = mine[j];
            const int y = who[j];
            mine[j] = mine[j - 1], who[j] = who[j - 1];
            mine[j - 1] = x, who[j - 1] = y;
          }
      unsigned long long bound = 0;
      for (int k = 0; k < K; ++k) {
        const uint32_t hi = static_cast<uint32_t>(mine[0] >> 32), top = __reduce_max_sync(0xffffffffu, hi);
        const uint32_t low = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(mine[0]) : 0u);
        bound = (static_cast<unsigned long long>(top) << 32) | low;
        const bool first = bound != 0 && mine[0] == bound;   // (fewer threads than K have vectors: all elements are looked at)
        if (lane == 0) s_who[k] = -1;
        __syncwarp();
        if (first) {
          s_who[k] = who[0];
#pragma unroll
          for (int i = 0; i + 1 < kEach; ++i) mine[i] = mine[i + 1], who[i] = who[i + 1];
          mine[kEach - 1] = 0;
        }
      }
      if (lane == 0) s_bound = bound;
    }
    __syncthreads();
    const unsigned long long bound = s_bound;
    const int steps = (v1 - v0 + kThreads - 1) / kThreads;
    for (int w = tid; w < K * steps; w += kThreads) {
      const int i = v0 + s_who[w % K] + w / K * kThreads;
      if (i < v0 || i >= v1) continue;
      float x[N];
      V16::unpack(row.load(i), x);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (key_of(x[e], static_cast<uint32_t>(i)) >= bound && row.has(i, e)) {
          const int at = atomicAdd(&s_n_found, 1);
          if (at < kMaxFound) s_found[at] = key_of(x[e], static_cast<uint32_t>(i * static_cast<long long>(N) + e - row.skip));
        }
      }
    }
    __syncthreads();
    const int n = s_n_found;
    if (n <= kMaxFound) {
      for (int c = tid; c < n; c += kThreads) {
        const unsigned long long key = s_found[c];
        int rank = 0;
        for (int o = 0; o < n; ++o) rank += s_found[o] > key ? 1 : 0;
        if (rank < K) s_best[rank] = key;
      }
    } else {
      unsigned long long last = ~0ull;
      for (int k = 0; k < K; ++k) {
        unsigned long long next = 0;
        for (int i = v0 + tid; i < v1; i += kThreads) {
          float x[N];
          V16::unpack(row.load(i), x);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const unsigned long long key = key_of(x[e], static_cast<uint32_t>(i * static_cast<long long>(N) + e - row.skip));
            if (row.has(i, e) && key < last && key > next) next = key;
          }
        }
        s_groups[tid] = next;
        __syncthreads();
        for (int d = kThreads / 2; d >= 1; d >>= 1) {
          if (tid < d) s_groups[tid] = max(s_groups[tid], s_groups[tid + d]);
          __syncthreads();
        }
        last = s_groups[0];
        if (tid == 0) s_best[k] = last;
        __syncthreads();
      }
    }
    __syncthreads();
  }

  // ---------------- the row's results ----------------
  if (p.parts > 1) {
    __syncwarp();
    cluster_sync();   // every part's sums and best are there
    if (part == 0) {
      if (tid == 0) {
        Sums t = s_part;
        for (int c = 1; c < p.parts; ++c) t = merge(t, *cluster_ptr(&s_part, c));
        s_part = t;
      }
      if constexpr (kTop) {
        const int n = p.parts * K;   // at most kMaxParts * kMaxTopLogprob
        static_assert(kMaxParts * kMaxTopLogprob <= kMaxFound, "the parts' best");
        for (int i = tid; i < n; i += kThreads) s_found[i] = *(cluster_ptr(s_best, i / K) + i % K);
        __syncthreads();
        if (tid < kMaxTopLogprob) s_best[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
          const unsigned long long key = s_found[i];
          int rank = 0;
          for (int o = 0; o < n; ++o) rank += s_found[o] > key ? 1 : 0;
          if (key != 0 && rank < K) s_best[rank] = key;
        }
        __syncthreads();
      }
    }
  }
  if (part == 0 && tid == 0) {
    const Sums t = s_part;
    const float log_s = logf(t.s), nan = __uint_as_float(0x7fc00000u);
    const bool none = t.s == 0.0f;
    p.lse[r] = none ? -INFINITY : t.m + log_s;
    p.entropy[r] = none ? nan : log_s - t.w * kLn2 / t.s;
    if (p.logp != nullptr) p.logp[r] = !has_tok ? 0.0f : none ? nan : (x_tok - t.m) - log_s;
    s_row = none ? make_float2(0.0f, nan) : make_float2(t.m, log_s);
  }
  if constexpr (kTop) {
    __syncthreads();
    if (part == 0) {
      for (int k = tid; k < p.topk; k += kThreads) {
        const bool some = k < K;
        p.top_idx[r * p.topk + k] = some ? static_cast<int32_t>(index_of(s_best[k])) : -1;
        p.top_logp[r * p.topk + k] = some ? (from_ordered(static_cast<uint32_t>(s_best[k] >> 32)) - s_row.x) - s_row.y : -INFINITY;
      }
    }
  }
  if (p.parts > 1) {
    __syncwarp();
    cluster_sync();   // no CTA leaves while it is read
  }
}

// Parts of a row, so that rows * parts CTAs fill the GPU's SMs `times` times over where a part has `least` vectors all the same. Rows alone do
// from 1216 on: 1 x 152064 bf16 take XX us in eight parts and XX in one.
int parts_of(int N, long long vecs, int times, long long least) {
  int parts = 1;
  while (parts < kMaxParts && static_cast<long long>(N) * parts < 152LL * times && vecs / (2 * parts) >= least) parts *= 2;
  return parts;
}

struct BwdParams {
  const void* logits;
  const int32_t* tok;
  const float* lse;
  const float* entropy;
  const float* d_logp;
  const float* d_entropy;
  const float* d_lse;
  const int32_t* top_idx;
  const float* d_top;
  void* out;
  int V, topk, parts;
};

// A CTA takes one of p.parts parts of a row's vectors. The elements that a token or an alternative names are read before the CTA writes
// any (the gradient may take the logits' place) and written again behind its vectors, with all that they get in one sum.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) logprob_bwd_kernel(const __grid_constant__ BwdParams p) {
  using V16 = Vec16<T>;
  constexpr int N = V16::kN, kInFlight = 4;
  __shared__ int s_idx[kMaxTopLogprob + 1];
  __shared__ float s_g[kMaxTopLogprob + 1];
  griddep_wait();
  griddep_launch_dependents();
  const int tid = threadIdx.x;
  const long long r = blockIdx.x / p.parts;
  const int part = static_cast<int>(blockIdx.x % p.parts);
  const Row<T> row(static_cast<const T*>(p.logits), r, p.V);
  const int each = (row.n_vecs + p.parts - 1) / p.parts;
  const int v0 = min(part * each, row.n_vecs), v1 = min(v0 + each, row.n_vecs);
  // named elements: the token, then the alternatives
  const int named = 1 + p.topk;
  int j = -1;
  float g = 0.0f;
  if (tid < named) {
    if (tid == 0) {
      if (p.tok != nullptr && p.d_logp != nullptr) j = __ldg(p.tok + r), g = __ldg(p.d_logp + r);
    } else {
      j = __ldg(p.top_idx + r * p.topk + tid - 1), g = __ldg(p.d_top + r * p.topk + tid - 1);
    }
    if (j < 0 || j >= p.V) j = -1, g = 0.0f;
    s_idx[tid] = j;
    s_g[tid] = g;
  }
  const float lse = __ldg(p.lse + r), g_h = p.d_entropy == nullptr ? 0.0f : __ldg(p.d_entropy + r);
  float x_named = 0.0f;
  const int vec = j < 0 ? -1 : static_cast<int>((static_cast<long long>(j) + row.skip) / N);
  const bool here = vec >= v0 && vec < v1;
  if (here) x_named = V16::value(static_cast<const T*>(p.logits)[r * p.V + j]);
  __syncthreads();
  float a = p.d_lse == nullptr ? 0.0f : __ldg(p.d_lse + r);
  for (int k = 0; k < named; ++k) a -= s_g[k];
  if (p.d_entropy != nullptr) a = fmaf(-g_h, __ldg(p.entropy + r), a);
  // p (a - g_h ln p), ln p = t ln 2
  const float b = g_h * kLn2;
  const auto plain = [&](float x) {
    const float t = max_nan((x - lse) * kLog2e, kFloor);
    return ex2_approx(t) * fmaf(-b, t, a);
  };
  T* out = static_cast<T*>(p.out) + r * p.V;
  uint4* vecs = reinterpret_cast<uint4*>(out - row.skip);
  const bool aligned = (reinterpret_cast<uintptr_t>(vecs) & 15) == 0;   // (else the outputs lie otherwise than the logits do)
  for (int i0 = v0 + tid; i0 < v1; i0 += kThreads * kInFlight) {
    uint4 raw[kInFlight];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const int i = i0 + k * kThreads;
      if (i < v1) raw[k] = row.whole(i) ? row.base[i] : row.load_end(i);
    }
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const int i = i0 + k * kThreads;
      if (i >= v1) break;
      float x[N];
      V16::unpack(raw[k], x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = plain(x[e]);
      if (aligned && row.whole(i)) {
        vecs[i] = V16::pack(x);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (row.has(i, e)) out[static_cast<long long>(i) * N + e - row.skip] = V16::from(x[e]);
      }
    }
  }
  __syncthreads();
  if (here) {
    float d = plain(x_named);
    for (int k = 0; k < named; ++k)
      if (s_idx[k] == j) d += s_g[k];
    out[j] = V16::from(d);
  }
}

}  // namespace

int launch_logprob_fwd(const LogprobArgs& a, cudaStream_t stream) {
  const long long vecs = (static_cast<long long>(a.V) * a.elem_bytes + 15) / 16;
  const int parts = parts_of(a.N, vecs, 8, 512);
  if (static_cast<long long>(a.N) * parts > 0x7fffffffLL) return -2;
  FwdParams p{a.logits, a.tok, a.logp, a.entropy, a.lse, a.top_idx, a.top_logp, a.V, a.topk, parts};
  cudaLaunchAttribute pdl[1], attr[2];
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(a.N * parts)), dim3(kThreads), 0, stream, pdl);
  if (parts > 1) {
    attr[0] = pdl[0];
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
  using bf16 = __nv_bfloat16;
  const auto fn = a.elem_bytes == 2 ? (a.topk > 0 ? logprob_fwd_kernel<bf16, true> : logprob_fwd_kernel<bf16, false>)
                                    : (a.topk > 0 ? logprob_fwd_kernel<float, true> : logprob_fwd_kernel<float, false>);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

int launch_logprob_bwd(const LogprobGradArgs& a, cudaStream_t stream) {
  const long long vecs = (static_cast<long long>(a.V) * a.elem_bytes + 15) / 16;
  const int parts = parts_of(a.N, vecs, 8, 512);
  if (static_cast<long long>(a.N) * parts > 0x7fffffffLL) return -2;
  BwdParams p{a.logits, a.tok, a.lse, a.entropy, a.d_logp, a.d_entropy, a.d_lse, a.top_idx, a.d_top, a.d_logits, a.V, a.topk, parts};
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(a.N * parts)), dim3(kThreads), 0, stream, attr);
  const cudaError_t e = a.elem_bytes == 2 ? cudaLaunchKernelEx(&cfg, logprob_bwd_kernel<__nv_bfloat16>, p)
                                          : cudaLaunchKernelEx(&cfg, logprob_bwd_kernel<float>, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
