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
// The K best. A thread keeps the best of its vectors (every 192nd) as (largest element, vector), of many the second best too, and the
// largest element of the others. The K-th best of the threads' best ones is a bound: every one of the K best elements lies in a vector whose
// pair is not behind it, and those are among the K threads in front. Their vectors are read again, the kept ones alone where the others'
// largest element is behind the bound, and the elements that are not behind it are ranked by counting. What passes the bound is little
// more than K, whatever ties there are (a row of equal logits: the first K vectors). A row whose K best crowd in a few threads may
// pass more than kMaxFound: then its vectors are all looked at again, once, and the bound rises with what is found.
//
// Bound by memory, and not far from it by the special-function units (an exponential an element: 56 us of the 76 that reading 2048 x
// 126464 bf16 takes). A CTA's warps have parts: six add up; one keeps a ring of three 12 KB pieces of the row's whole vectors filled by
// bulk copies, and runs on into the CTA's next row; one puts a row's sums and K best together while the others are at the next row
// (together with them that took 17 us of 113 for 8 alternatives, 35 for 20). Four CTAs share an SM. Vectors at the row's ends are loaded by
// two threads. Few rows are split over the CTAs of a cluster, whose sums and K best its first CTA puts together.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cluster.cuh"
#include "context.cuh"
#include "kernels.cuh"
#include "ptx.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxFound = 768;         // elements ranked at once
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -1000.0f;     // log2 units: 2^kFloor is 0, and 0 * kFloor too (0 * -inf is not)
constexpr float kSlack = 6.0f;         // the reference follows maxima that are above it by more
constexpr int kMaxParts = 8;           // of a row: CTAs of a cluster
// the forward kernel's warps: those that add up, one that copies, one that finishes rows
constexpr int kAddWarps = 6, kCopyWarp = 6, kAdders = 32 * kAddWarps, kFwdThreads = kAdders + 64;
constexpr int kEach = 4, kPiece = kEach * kAdders, kStages = 3;   // vectors of a thread, of a piece; pieces in flight

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
  static __device__ __forceinline__ float at(const uint4& r, int e) {
    const uint32_t w = e < 4 ? (e < 2 ? r.x : r.y) : (e < 6 ? r.z : r.w);
    return __uint_as_float((e & 1) != 0 ? w & 0xffff0000u : w << 16);
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
  static __device__ __forceinline__ float at(const uint4& r, int e) { return __uint_as_float(e < 2 ? (e < 1 ? r.x : r.y) : (e < 3 ? r.z : r.w)); }
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
  // the whole vectors x .. y - 1 of one of `parts` parts
  __device__ __forceinline__ int2 part(int i, int parts) const {
    const int each = (n_vecs + parts - 1) / parts, v0 = min(i * each, n_vecs), v1 = min(v0 + each, n_vecs), w0 = max(v0, whole0);
    return make_int2(w0, max(w0, min(v1, whole1)));
  }
  // whether element e of vector i is in the row
  __device__ __forceinline__ bool has(int i, int e) const {
    const long long j = static_cast<long long>(i) * Vec16<T>::kN + e - skip;
    return j >= 0 && j < V;
  }
  // whether vector i, the row's first (side 0) or last, is one of the part's and not whole
  __device__ __forceinline__ bool is_end(int i, int side, int k, int parts) const {
    const int each = (n_vecs + parts - 1) / parts, v0 = min(k * each, n_vecs), v1 = min(v0 + each, n_vecs);
    return i >= v0 && i < v1 && !whole(i) && (side == 0 || i > 0);
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

__device__ __forceinline__ bool warp_wait_all(uint64_t* bar, uint32_t parity, const volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

struct FwdParams {
  const void* logits;
  const int32_t* tok;
  float* logp;
  float* entropy;
  float* lse;
  int32_t* top_idx;
  float* top_logp;
  int* status;
  int N, V, topk, parts;
};

// A thread's sums for logits of any size: over whole vectors w0 + tid, w0 + tid + kAdders, .. below w1, and one at the row's ends.
template <typename T>
__device__ __noinline__ Sums careful_sums(const Row<T>& row, int w0, int w1, bool has_end, uint4 end_raw) {
  constexpr int N = Vec16<T>::kN;
  Sums a{-INFINITY, 0.0f, 0.0f};
  const auto add = [&](const uint4& raw) {
    float x[N];
    Vec16<T>::unpack(raw, x);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (x[e] == -INFINITY) continue;
      const float t = max_nan((x[e] - a.m) * kLog2e, kFloor), f = ex2_approx(t);
      a.s += f;
      a.w = fmaf(f, t, a.w);
    }
  };
  for (int k = w0 + threadIdx.x; k < w1; k += kAdders) a.m = fmaxf(a.m, Vec16<T>::top(__ldg(row.base + k)));
  if (has_end) a.m = fmaxf(a.m, Vec16<T>::top(end_raw));
  for (int k = w0 + threadIdx.x; k < w1; k += kAdders) add(__ldg(row.base + k));
  if (has_end) add(end_raw);
  return a;
}

// Alternatives asked for: none, up to kFewBest, or more. For few the threads' best vectors are enough, and the K best of the threads are taken
// one after the other. For more, threads with two or three of the best ones are no exception and taking is slow: a thread keeps two vectors
// and the bound is found by halving. Measured the first / second way, 2048 rows of 126464 bf16: 1 alternative 87 / 100 us, 5 88 / 100, 16 94 / 100,
// 20 102 / 101, 64 251 / 126; 972 of 25063: 19 / 22, 21 / 23, 24 / 24, 26 / 24, 58 / 34; one of 32000: 6.4 / 7.8, 7.5 / 8.3, 10.9 / 8.9, 11.9 / 9.1,
// 29 / 17. (Single rows would change ways at 8 alternatives, batches do at 20.)
enum Best { kNone, kFew, kMany };
constexpr int kFewBest = 16;

// A row's sums and pairs, from the adding warps to the finishing one.
template <Best kBest>
struct Handover {
  Sums sums[kAddWarps];
  unsigned long long pairs[kBest == kMany ? 2 : 1][kBest != kNone ? kAdders : 1];   // a thread's best vector, or its two best
  float others[kBest != kNone ? kAdders : 1];                                       // the largest element of its other vectors
};

template <Best kBest>
struct FwdShared {
  uint64_t full[kStages], empty[kStages], done[2], taken[2];
  Handover<kBest> row[2];
  Sums part;                          // the finishing warp's, read by the cluster's first CTA
  unsigned long long best[kBest != kNone ? kMaxTopLogprob : 1];
  unsigned long long found[kBest != kNone ? kMaxFound : 1];
  int who[kBest != kNone ? 2 * kMaxTopLogprob : 1], more[kBest != kNone ? kMaxTopLogprob : 1];
  int n_found, abort;
};

// The K best of sorted lists, one a lane (`next(i)`: its i-th key, 0 behind the end), in order: take(k, key) by all lanes. Returns the last.
template <typename Next, typename Take>
__device__ __forceinline__ unsigned long long merge_best(int K, Next&& next, Take&& take) {
  int at = 0;
  unsigned long long mine = next(0), last = 0;
  for (int k = 0; k < K; ++k) {
    const uint32_t hi = static_cast<uint32_t>(mine >> 32), top = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t low = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(mine) : 0u);
    last = (static_cast<unsigned long long>(top) << 32) | low;
    take(k, last);
    if (mine == last && last != 0) mine = next(++at);
  }
  return last;
}

// A bound that K to K + K / 4 of a warp's keys, and at most kMaxTopLogprob, are not below (kLists keys a lane), found by halving, the values
// first (the upper kBits of a key), then the indices of the keys of the value that is cut; 0 where there are fewer than K keys. (Exactly K: the 20
// best of one row of 32000 took 0.8 us more; what is looked at besides costs 2048 rows of 126464 1 %.)
template <int kBits, int kLists>
__device__ __forceinline__ unsigned long long bound_of(const unsigned long long (&keys)[kLists], int K) {
  const int most = min(K + K / 4, kMaxTopLogprob);
  const auto upper = [](unsigned long long key) { return static_cast<uint32_t>(key >> (64 - kBits)); };
  // the lowest key of a value (the lower half of the word of a bf16 is zeros, or ones where it is negative)
  const auto of_value = [](uint32_t u) {
    const uint32_t word = kBits == 32 ? u : (u << 16) | ((u & 0x8000u) != 0 ? 0u : 0xffffu);
    return static_cast<unsigned long long>(word) << 32;
  };
  uint32_t hi = 0, lo = 0xffffffffu;
  int n = 0;
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    if (keys[i] == 0) continue;
    hi = max(hi, upper(keys[i])), lo = min(lo, upper(keys[i])), ++n;
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if (n < K) return 0;
  hi = __reduce_max_sync(0xffffffffu, hi), lo = __reduce_min_sync(0xffffffffu, lo);
  // moves `from` up to the last start of `least` or more; n: how many that is
  const auto halve = [&](uint32_t& from, uint32_t to, int least, int enough, auto&& is) {
    while (from < to && n > enough) {
      const uint32_t mid = from + (to - from + 1) / 2;
      int c = 0;
#pragma unroll
      for (int i = 0; i < kLists; ++i) c += is(keys[i], mid) ? 1 : 0;
      c = __reduce_add_sync(0xffffffffu, c);
      if (c >= least) from = mid, n = c;
      else to = mid - 1;
    }
  };
  halve(lo, hi, K, most, [&](unsigned long long key, uint32_t mid) { return upper(key) >= mid; });
  const unsigned long long value = of_value(lo);
  if (n <= most) return value;
  // too many are of value lo
  int above = 0, ties = 0;
  uint32_t first = 0xffffffffu, last = 0;
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    above += upper(keys[i]) > lo ? 1 : 0;
    if (keys[i] == 0 || upper(keys[i]) != lo) continue;
    const uint32_t low = static_cast<uint32_t>(keys[i]);
    first = min(first, low), last = max(last, low), ++ties;
  }
  above = __reduce_add_sync(0xffffffffu, above), n = __reduce_add_sync(0xffffffffu, ties);
  first = __reduce_min_sync(0xffffffffu, first), last = __reduce_max_sync(0xffffffffu, last);
  halve(first, last, K - above, most - above, [&](unsigned long long key, uint32_t mid) {
    return upper(key) == lo && key != 0 && static_cast<uint32_t>(key) >= mid;
  });
  return value | first;
}

// Puts the n keys of `from` in order, the K best of them into `to`: a key's place is the number of those in front of it.
__device__ __forceinline__ void rank_keys(const unsigned long long* from, int n, int K, unsigned long long* to, int lane) {
  for (int c = lane; c < n; c += 32) {
    const unsigned long long key = from[c];
    int rank = 0;
    for (int o = 0; o < n; ++o) rank += from[o] > key ? 1 : 0;
    if (rank < K) to[rank] = key;
  }
}

// The K best of a part's elements, where more of them than are ranked at once are not below `least` (-inf: any may be). One walk over the part's
// vectors, by a warp: what is not behind the bound is kept, and where there may be no room for the next vectors' the bound rises to one
// that K of the kept, or little more, are not behind. However the logits lie, that is one look at each and at most one rise for 192 kept. (A walk for
// each alternative takes K times as long, and in rows of several million logits longer than the other warps wait.) Returns how many are in `found`.
constexpr int kKept = 512;
static_assert(kKept <= kMaxFound && kKept >= kMaxTopLogprob + 256, "room for a vector a lane behind those that stay");
template <typename T>
__device__ __forceinline__ int find_crowded(const Row<T>& row, int part, int parts, int K, float least, unsigned long long* found) {
  using V16 = Vec16<T>;
  constexpr int N = V16::kN;
  const int2 w = row.part(part, parts);
  const int lane = threadIdx.x & 31, most = min(K + K / 4, kMaxTopLogprob);
  const uint32_t before = (1u << lane) - 1u;
  unsigned long long bound = least == -INFINITY ? 0 : static_cast<unsigned long long>(ordered(least)) << 32;
  int n = 0;
  const auto rise = [&] {
    __syncwarp();
    // the bound is one of the keys (no two are the same), tried in turn: from one that the middle of the lanes holds between those that let
    // too many through and those that let too few
    unsigned long long above = ~0ull, key = found[n / 2];
    for (int here = n; here > most;) {
      int c = 0;
      unsigned long long low = 0, high = 0;
#pragma unroll 1
      for (int k = lane; k < n; k += 32) {
        const unsigned long long x = found[k];
        c += x >= key ? 1 : 0;
        if (x > key && x < above) high = x;
        if (x < key && x > bound) low = x;
      }
      c = __reduce_add_sync(0xffffffffu, c);
      if (c >= K) bound = key, here = c;
      else above = key;
      const unsigned long long mine = c >= K ? high : low;
      const uint32_t lanes = __ballot_sync(0xffffffffu, mine != 0);
      const uint32_t middle = __ballot_sync(0xffffffffu, mine != 0 && __popc(lanes & before) == __popc(lanes) / 2);
      key = __shfl_sync(0xffffffffu, mine, __ffs(middle) - 1);
    }
    least = from_ordered(static_cast<uint32_t>(bound >> 32));
    const int all = n;
    n = 0;
    for (int k = 0; k < all; k += 32) {
      const unsigned long long key = k + lane < all ? found[k + lane] : 0;
      const bool in = key >= bound && key != 0;
      const uint32_t lanes = __ballot_sync(0xffffffffu, in);
      if (in) found[n + __popc(lanes & before)] = key;   // (a place that has been read)
      n += __popc(lanes);
      __syncwarp();
    }
  };
  const auto keep = [&](bool there, const uint4& raw, int i) {   // a vector a lane
    const bool some = there && !(V16::top(raw) < least);
    if (!__any_sync(0xffffffffu, some)) return;
    if (n > kKept - 32 * N) rise();
#pragma unroll 1
    for (int e = 0; e < N; ++e) {
      const uint32_t j = static_cast<uint32_t>(i) * N + e - row.skip;   // (above V where it is another row's)
      const unsigned long long key = key_of(V16::at(raw, e), j);
      const bool in = some && key >= bound && j < static_cast<uint32_t>(row.V);
      const uint32_t lanes = __ballot_sync(0xffffffffu, in);
      if (in) found[n + __popc(lanes & before)] = key;
      n += __popc(lanes);
    }
  };
  const int end = lane == 0 ? 0 : row.n_vecs - 1;
  const bool is_end = lane < 2 && row.is_end(end, lane, part, parts);
#pragma unroll 1
  for (int i0 = w.x;; i0 += 32) {
    const bool ends = i0 >= w.y, there = ends ? is_end : i0 + lane < w.y;
    const int i = ends ? end : i0 + lane;
    keep(there, there ? row.load(i) : make_uint4(0, 0, 0, 0), i);
    if (ends) break;
  }
  __syncwarp();
  return n;
}

template <typename T, Best kBest>
__global__ void __launch_bounds__(kFwdThreads, 4) logprob_fwd_kernel(const __grid_constant__ FwdParams p) {
  using V16 = Vec16<T>;
  constexpr int N = V16::kN;
  extern __shared__ uint4 ring[];   // [kStages][kPiece]
  constexpr bool kTop = kBest != kNone;
  __shared__ FwdShared<kBest> sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = p.parts > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], kAddWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.done[i], kAddWarps);
      mbar_init(&sm.taken[i], 1);
    }
    sm.abort = 0;
    fence_mbar_init();
  }
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const int first_row = blockIdx.x / p.parts, row_step = p.parts > 1 ? p.N : static_cast<int>(gridDim.x);

  if (warp == kCopyWarp) {
    // ---------------- copies ----------------
    if (lane == 0) {
      int piece = 0;
      bool ok = true;
      for (long long r = first_row; r < p.N && ok; r += row_step) {
        const Row<T> row(static_cast<const T*>(p.logits), r, p.V);
        const int2 w = row.part(part, p.parts);
        for (int v = w.x; v < w.y && ok; v += kPiece, ++piece) {
          const int st = piece % kStages;
          if (piece >= kStages) ok = mbar_wait(&sm.empty[st], (piece / kStages - 1) & 1, &sm.abort);
          if (!ok) break;
          const uint32_t bytes = static_cast<uint32_t>(min(kPiece, w.y - v)) * 16;
          mbar_arrive_expect_tx(&sm.full[st], bytes);
          bulk_load(smem_u32(ring + st * kPiece), row.base + v, bytes, &sm.full[st]);
        }
      }
      if (!ok) {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 90);
        sm.abort = 1;
      }
      // every copy lands before the CTA's shared memory is released, whatever the other warps did
      for (int f = max(0, piece - kStages); f < piece; ++f) mbar_wait(&sm.full[f % kStages], (f / kStages) & 1, nullptr);
    }
    __syncwarp();
  } else if (warp < kAddWarps) {
    // ---------------- sums, and each thread's best vector ----------------
    int piece = 0, n_row = 0;
    bool ok = true;
    for (long long r = first_row; r < p.N && ok; r += row_step, ++n_row) {
      const Row<T> row(static_cast<const T*>(p.logits), r, p.V);
      const int2 w = row.part(part, p.parts);
      const int end = tid == 0 ? 0 : row.n_vecs - 1;
      const bool has_end = tid < 2 && row.is_end(end, tid, part, p.parts);
      uint4 end_raw = make_uint4(0, 0, 0, 0);
      if (has_end) end_raw = row.load_end(end);
      Sums a{-INFINITY, 0.0f, 0.0f};
      bool careful = false;
      float c = -INFINITY;
      uint32_t floor = 0;
      uint64_t s2[2] = {0, 0}, w2[2] = {0, 0};
      float best[2] = {-INFINITY, -INFINITY}, others = -INFINITY;
      int best_vec[2] = {w.x + tid, 0};
      const auto take = [&](const auto& raw, auto count, int i0) {
        constexpr int n = decltype(count)::value;
        float top = -INFINITY, t[n];
#pragma unroll
        for (int k = 0; k < n; ++k) {
          t[k] = V16::top(raw[k]);
          top = fmaxf(top, t[k]);
        }
        if constexpr (kBest == kFew) {
          if (top > best[0]) {
            others = fmaxf(others, best[0]);
            best[0] = top;
            bool found = false;
#pragma unroll
            for (int k = 0; k < n; ++k) {
              const bool this_one = !found && t[k] == top;
              if (this_one) best_vec[0] = i0 + k * kAdders;
              else others = fmaxf(others, t[k]);
              found |= this_one;
            }
          } else {
            others = fmaxf(others, top);
          }
        } else if constexpr (kBest == kMany) {
          if (top > best[1]) {
#pragma unroll
            for (int k = 0; k < n; ++k) {
              const int vec = i0 + k * kAdders;
              if (t[k] > best[0]) {
                others = fmaxf(others, best[1]);
                best[1] = best[0], best_vec[1] = best_vec[0];
                best[0] = t[k], best_vec[0] = vec;
              } else if (t[k] > best[1]) {
                others = fmaxf(others, best[1]);
                best[1] = t[k], best_vec[1] = vec;
              } else {
                others = fmaxf(others, t[k]);
              }
            }
          } else {
            others = fmaxf(others, top);
          }
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
          for (int k = 0; k < n; ++k) {
            float x[N];
            V16::unpack(raw[k], x);
#pragma unroll
            for (int e = 0; e < N; ++e) careful |= x[e] != x[e];
          }
          return;
        }
        const uint64_t l2 = f2_pack(kLog2e, kLog2e), c2 = f2_pack(-c, -c);
#pragma unroll
        for (int k = 0; k < n; ++k) {
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
      };
      using Many = std::integral_constant<int, kEach>;
      using One = std::integral_constant<int, 1>;
      for (int v = w.x; v < w.y; v += kPiece, ++piece) {
        const int st = piece % kStages;
        ok = warp_wait_all(&sm.full[st], (piece / kStages) & 1, &sm.abort);
        if (!ok) break;
        const uint4* vecs = ring + st * kPiece + tid;
        if (v + kPiece <= w.y) {
          uint4 raw[kEach];
#pragma unroll
          for (int k = 0; k < kEach; ++k) raw[k] = vecs[k * kAdders];
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.empty[st]);
          take(raw, Many{}, v + tid);
        } else {
          for (int i = v + tid; i < w.y; i += kAdders, vecs += kAdders) {
            const uint4 one[1] = {*vecs};
            take(one, One{}, i);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.empty[st]);
        }
      }
      const int buf = n_row & 1;
      if (ok && n_row >= 2) ok = warp_wait_all(&sm.taken[buf], ((n_row >> 1) - 1) & 1, &sm.abort);
      if (!ok) break;
      if constexpr (kTop) {
        sm.row[buf].pairs[0][tid] = w.x + tid < w.y ? key_of(best[0], static_cast<uint32_t>(best_vec[0])) : 0ull;
        // (a second of -inf alone is left to the walk over the others, which are no less)
        if constexpr (kBest == kMany) sm.row[buf].pairs[1][tid] = best[1] > -INFINITY ? key_of(best[1], static_cast<uint32_t>(best_vec[1])) : 0ull;
        sm.row[buf].others[tid] = others;
      }
      // the row's ends are no thread's pairs (they are looked at anyway)
      if (has_end) {
        const uint4 one[1] = {end_raw};
        take(one, One{}, end);
      }
      if (careful) {
        a = careful_sums(row, w.x, w.y, has_end, end_raw);
      } else if (a.m != -INFINITY) {
        float x[4];
        f2_unpack(f2_add(s2[0], s2[1]), x[0], x[1]);
        f2_unpack(f2_add(w2[0], w2[1]), x[2], x[3]);
        const float off = fmaf(a.m, kLog2e, -c), f = ex2_approx(-off);
        a.s = (x[0] + x[1]) * f;
        a.w = fmaf(-off, x[0] + x[1], x[2] + x[3]) * f;
      }
      float to = a.m;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, d));
      a.move_to(to);
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, d);
      }
      if (lane == 0) sm.row[buf].sums[warp] = a;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.done[buf]);
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 91);
      sm.abort = 1;
    }
  } else {
    // ---------------- the rows' results ----------------
    const int K = kTop ? min(p.topk, p.V) : 0;
    int n_row = 0;
    bool ok = true;
    Sums all{-INFINITY, 0.0f, 0.0f};
    float x_tok = 0.0f;
    bool has_tok = false;
    const auto write = [&](long long r) {
      const float log_s = logf(all.s), nan = __uint_as_float(0x7fc00000u);
      const bool none = all.s == 0.0f;
      if (lane == 0) {
        p.lse[r] = none ? -INFINITY : all.m + log_s;
        p.entropy[r] = none ? nan : log_s - all.w * kLn2 / all.s;
        if (p.logp != nullptr) p.logp[r] = !has_tok ? 0.0f : none ? nan : (x_tok - all.m) - log_s;
      }
      if constexpr (kTop) {
        for (int k = lane; k < p.topk; k += 32) {
          const bool some = k < K;
          const unsigned long long key = some ? sm.best[k] : 0;
          p.top_idx[r * p.topk + k] = some ? static_cast<int32_t>(index_of(key)) : -1;
          p.top_logp[r * p.topk + k] = !some ? -INFINITY : none ? nan : (from_ordered(static_cast<uint32_t>(key >> 32)) - all.m) - log_s;
        }
      }
    };
    for (long long r = first_row; r < p.N && ok; r += row_step, ++n_row) {
      const Row<T> row(static_cast<const T*>(p.logits), r, p.V);
      const int2 w = row.part(part, p.parts);
      has_tok = false;
      if (part == 0 && p.tok != nullptr) {
        const int y = __ldg(p.tok + r);
        has_tok = y >= 0 && y < p.V;
        if (has_tok) x_tok = V16::value(static_cast<const T*>(p.logits)[r * p.V + y]);
      }
      const int buf = n_row & 1;
      ok = warp_wait_all(&sm.done[buf], (n_row >> 1) & 1, &sm.abort);
      if (!ok) break;
      all = sm.row[buf].sums[0];
#pragma unroll
      for (int i = 1; i < kAddWarps; ++i) all = merge(all, sm.row[buf].sums[i]);
      if constexpr (kTop) {
        constexpr int kLists = kAdders / 32;
        // the K best pairs
        unsigned long long mine[kLists];
#pragma unroll
        for (int i = 0; i < kLists; ++i) mine[i] = sm.row[buf].pairs[0][32 * i + lane];
        if (lane == 0) sm.n_found = 0;
        for (int k = lane; k < kMaxTopLogprob; k += 32) sm.best[k] = 0;   // (NaN may leave places empty)
        // (where fewer threads than K have vectors the bound is 0, and all their elements are looked at)
        unsigned long long bound;
        float bound_value;
        int n_who = 0, n_more = 0;
        const uint32_t before = (1u << lane) - 1u;
        if constexpr (kBest == kFew) {
          // a lane's, in order
#pragma unroll
          for (int i = 1; i < kLists; ++i)
#pragma unroll
            for (int j = i; j > 0; --j) {
              const unsigned long long hi = max(mine[j - 1], mine[j]), lo = min(mine[j - 1], mine[j]);
              mine[j - 1] = hi, mine[j] = lo;
            }
          const auto next = [&](int i) {
            unsigned long long key = 0;
#pragma unroll
            for (int k = 0; k < kLists; ++k)
              if (i == k) key = mine[k];
            return key;
          };
          bound = merge_best(K, next, [&](int k, unsigned long long key) {
            if (lane == 0 && key != 0) sm.who[k] = static_cast<int>(index_of(key));
            if (key != 0) n_who = k + 1;
          });
          bound_value = from_ordered(static_cast<uint32_t>(bound >> 32));
          __syncwarp();
          static_assert(kFewBest <= 32, "a thread's vector a lane");
          const int t = lane < n_who ? (sm.who[lane] - w.x) % kAdders : 0;
          const bool more = lane < n_who && (bound == 0 || !(sm.row[buf].others[t] < bound_value));
          const uint32_t walk = __ballot_sync(0xffffffffu, more);
          if (more) sm.more[__popc(walk & before)] = t;
          n_more = __popc(walk);
        } else {
          bound = bound_of<8 * sizeof(T)>(mine, K);
          bound_value = from_ordered(static_cast<uint32_t>(bound >> 32));
#pragma unroll
          for (int i = 0; i < kLists; ++i) {
            const unsigned long long second = sm.row[buf].pairs[1][32 * i + lane];
            const bool in = mine[i] != 0 && mine[i] >= bound, in2 = in && second != 0 && second >= bound;
            const bool more = in && (bound == 0 || !(sm.row[buf].others[32 * i + lane] < bound_value));
            const uint32_t lanes = __ballot_sync(0xffffffffu, in), lanes2 = __ballot_sync(0xffffffffu, in2), walk = __ballot_sync(0xffffffffu, more);
            if (in) sm.who[n_who + __popc(lanes & before)] = static_cast<int>(index_of(mine[i]));
            n_who += __popc(lanes);
            if (in2) sm.who[n_who + __popc(lanes2 & before)] = static_cast<int>(index_of(second));
            n_who += __popc(lanes2);
            if (more) sm.more[n_more + __popc(walk & before)] = 32 * i + lane;
            n_more += __popc(walk);
          }
        }
        __syncwarp();
        const auto look = [&](const uint4& raw, int i) {
          if (bound != 0 && V16::top(raw) < bound_value) return;
          float x[N];
          V16::unpack(raw, x);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            if (bound != 0 && x[e] < bound_value) continue;
            if (key_of(x[e], static_cast<uint32_t>(i)) >= bound && row.has(i, e)) {
              const int at = atomicAdd(&sm.n_found, 1);
              if (at < kMaxFound) sm.found[at] = key_of(x[e], static_cast<uint32_t>(i * static_cast<long long>(N) + e - row.skip));
            }
          }
        };
        for (int k = lane; k < n_who; k += 32) look(__ldg(row.base + sm.who[k]), sm.who[k]);
        // threads whose other vectors may hold some too: these are dealt out to the lanes, kLooked loads at a time (a thread after the other
        // 64 alternatives of 128k logits took 20 us)
        constexpr int kLooked = 4;
        const int each = (w.y - w.x + kAdders - 1) / kAdders, todo = n_more * each;
        int m = lane / max(each, 1), step = lane - m * each;   // a lane's place: the thread's in the list, the vector's among its
        for (int i0 = lane; i0 < todo; i0 += 32 * kLooked) {
          uint4 raw[kLooked];
          int at[kLooked];
#pragma unroll
          for (int u = 0; u < kLooked; ++u) {
            at[u] = -1;
            if (i0 + 32 * u < todo) {
              const int t = sm.more[m], x = w.x + t + step * kAdders;
              const bool seen = x == static_cast<int>(index_of(sm.row[buf].pairs[0][t])) ||
                                (kBest == kMany && sm.row[buf].pairs[kBest == kMany ? 1 : 0][t] != 0 &&
                                 x == static_cast<int>(index_of(sm.row[buf].pairs[kBest == kMany ? 1 : 0][t])));
              if (x < w.y && !seen) {
                at[u] = x;
                raw[u] = __ldg(row.base + x);
              }
            }
            for (step += 32; step >= each; step -= each) ++m;
          }
#pragma unroll
          for (int u = 0; u < kLooked; ++u)
            if (at[u] >= 0) look(raw[u], at[u]);
        }
        if (lane < 2) {
          const int end = lane == 0 ? 0 : row.n_vecs - 1;
          if (row.is_end(end, lane, part, p.parts)) look(row.load_end(end), end);
        }
        __syncwarp();
        int n = sm.n_found;
        if (__builtin_expect(n > kMaxFound, 0)) {
          // (the row is put together anew from numbers that the compiler does not know again: kept over this walk, it spilled registers where every
          // row passes, and 2048 rows of 126464 with 8 alternatives took 92 us, not 90)
          long long again = r;
          int V = p.V;
          asm volatile("" : "+l"(again), "+r"(V));
          const Row<T> same(static_cast<const T*>(p.logits), again, V);
          n = find_crowded(same, part, p.parts, K, bound == 0 ? -INFINITY : bound_value, sm.found);
        }
        rank_keys(sm.found, n, K, sm.best, lane);
      }
      __syncwarp();
      if (p.parts == 1) write(r);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.taken[buf]);
    }
    if (lane == 0) sm.part = all;
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 92);
      sm.abort = 1;
    }
    if (p.parts > 1) {
      __syncwarp();
      cluster_sync();   // every part's sums and best are there
      if (part == 0 && ok) {
        for (int c = 1; c < p.parts; ++c) all = merge(all, *cluster_ptr(&sm.part, c));
        if constexpr (kTop) {
          static_assert(kMaxParts * kMaxTopLogprob <= kMaxFound, "the parts' best");
          if constexpr (kBest == kFew) {
            // the parts' lists, which are in order: brought here, then merged, one a lane
            for (int i = lane; i < p.parts * K; i += 32) sm.found[i] = cluster_ptr(sm.best, i / K)[i % K];
            __syncwarp();
            merge_best(K, [&](int i) { return lane < p.parts && i < K ? sm.found[lane * K + i] : 0ull; },
                       [&](int k, unsigned long long key) {
                         if (lane == 0) sm.best[k] = key;
                       });
          } else {
            // the parts' lists: K of their keys or little more, ranked (held in six keys a lane where that is enough: with sixteen, mostly
            // none, the 20 best of one row of 152064 took 11.7 us, so 10.7)
            int n = 0;
            const auto pick = [&](auto lists) {
              constexpr int kLists = decltype(lists)::value;
              unsigned long long theirs[kLists];
#pragma unroll
              for (int i = 0; i < kLists; ++i) {
                const int at = 32 * i + lane;
                theirs[i] = at < p.parts * K ? cluster_ptr(sm.best, at / K)[at % K] : 0ull;
              }
              const unsigned long long bound = bound_of<8 * sizeof(T)>(theirs, K);
#pragma unroll
              for (int i = 0; i < kLists; ++i) {
                const bool in = theirs[i] != 0 && theirs[i] >= bound;
                const uint32_t lanes = __ballot_sync(0xffffffffu, in);
                if (in) sm.found[n + __popc(lanes & ((1u << lane) - 1u))] = theirs[i];
                n += __popc(lanes);
              }
            };
            if (p.parts * K <= 6 * 32) pick(std::integral_constant<int, 6>{});
            else pick(std::integral_constant<int, kMaxParts * kMaxTopLogprob / 32>{});
            __syncwarp();
            for (int k = n + lane; k < K; k += 32) sm.best[k] = 0;
            rank_keys(sm.found, n, K, sm.best, lane);
          }
          __syncwarp();
        }
        write(first_row);
      }
      __syncwarp();
      cluster_sync();   // no CTA leaves while it is read
    }
    return;
  }
  if (p.parts > 1) {
    __syncwarp();
    cluster_sync();
    cluster_sync();
  }
}

// Parts of a row: as many, a power of two, as keep rows * parts at or below `times` CTAs an SM and leave a part `least` vectors.
int parts_of(int N, long long vecs, int times, long long least) {
  int parts = 1;
  while (parts < kMaxParts && 2LL * N * parts <= 152LL * times && vecs / (2 * parts) >= least) parts *= 2;
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

int launch_logprob_fwd(const LogprobArgs& a, int* status, cudaStream_t stream) {
  constexpr int kRingBytes = kStages * kPiece * 16;
  const long long vecs = (static_cast<long long>(a.V) * a.elem_bytes + 15) / 16;
  const int parts = parts_of(a.N, vecs, 4, 512);
  FwdParams p{a.logits, a.tok, a.logp, a.entropy, a.lse, a.top_idx, a.top_logp, status, a.N, a.V, a.topk, parts};
  // rows that are not split: as many CTAs as the GPU holds at once, one row after the other each
  const int ctas = parts > 1 ? a.N * parts : std::min(a.N, 4 * 152);
  cudaLaunchAttribute pdl[1], attr[2];
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(ctas)), dim3(kFwdThreads), kRingBytes, stream, pdl);
  if (parts > 1) {
    attr[0] = pdl[0];
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
  using bf16 = __nv_bfloat16;
  static ContextCache<int> setup;   // with the static part of a kernel with alternatives the ring is more than 48 KB
  int unused = 0;
  const int rc = setup.get(&unused, [](int&) {
    const auto allow = [](auto fn) { return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes) == cudaSuccess; };
    return allow(logprob_fwd_kernel<bf16, kFew>) && allow(logprob_fwd_kernel<bf16, kMany>) && allow(logprob_fwd_kernel<float, kFew>) &&
                   allow(logprob_fwd_kernel<float, kMany>)
               ? 0
               : -3;
  });
  if (rc != 0) return rc;
  const auto of = [&](auto zero) {
    using T = decltype(zero);
    return a.topk == 0 ? logprob_fwd_kernel<T, kNone> : a.topk <= kFewBest ? logprob_fwd_kernel<T, kFew> : logprob_fwd_kernel<T, kMany>;
  };
  const auto fn = a.elem_bytes == 2 ? of(bf16{}) : of(0.0f);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

int launch_logprob_bwd(const LogprobGradArgs& a, cudaStream_t stream) {
  const long long vecs = (static_cast<long long>(a.V) * a.elem_bytes + 15) / 16;
  const int parts = parts_of(a.N, vecs, 12, 512);
  if (static_cast<long long>(a.N) * parts > 0x7fffffffLL) return -2;
  BwdParams p{a.logits, a.tok, a.lse, a.entropy, a.d_logp, a.d_entropy, a.d_lse, a.top_idx, a.d_top, a.d_logits, a.V, a.topk, parts};
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(a.N * parts)), dim3(kThreads), 0, stream, attr);
  const cudaError_t e = a.elem_bytes == 2 ? cudaLaunchKernelEx(&cfg, logprob_bwd_kernel<__nv_bfloat16>, p)
                                          : cudaLaunchKernelEx(&cfg, logprob_bwd_kernel<float>, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
