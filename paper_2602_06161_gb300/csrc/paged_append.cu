// paged_append.cu - new rows of keys and values into a memory in pages, rotated to their positions on the way.
//
// k_pages, v_pages [n_pages, Hkv, page, D] bf16; position t of sequence b is row t % page of the page table[b, t / page].
// Row s of sequence b goes to start[b] + s (s < count[b]), or to pos[b, s], where of rows that name one position the
// lowest is taken; what has no page (a position outside the table, an entry outside the pool) is left out. k, and q beside
// it, turn by their positions first (the formulas and the angles of rope_kernel.cu), in fp32, and are rounded once.
//
// Bound by memory: every row is read and written once. Work is dealt out as in rope_kernel.cu: a thread holds one 16-byte vector column (two,
// R / 2 apart, in the layout of halves) of one token and walks over up to eight heads of q, k or v, so that its sines and
// cosines, and its token's place, serve all of them.
#include <cuda_bf16.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;
using bf16 = __nv_bfloat16;

struct AppendTensor {
  const uint8_t* in;
  uint8_t* out;      // dense rows [B, heads, n, D], or null
  bf16* pages;       // or null (q)
  long long in_b, in_h, in_l;   // strides in elements
  int heads, chunks;
};

struct AppendParams {
  AppendTensor t[3];        // q, k, v
  const double* inv_freq;   // [R / 2] radians per position
  const int32_t* table;
  const int32_t* start;     // [B], or null: pos
  const int32_t* count;     // [B] or null
  const int32_t* pos;       // [B, n]
  const int32_t* rope_pos;  // [B, n] or null: the row's position in the memory
  int n, D, R, M, n_pages, page_log2, Hkv;
  int units, turn_units;    // a row's work items; of them, those that turn
  int chunks;
  long long items;
  float mscale;
};

// T: element of the rows; N: elements of a thread's vector (16 bytes, or one element); kInter: pairs of neighbours.
template <typename T, int N, bool kInter>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) paged_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int kHeadsInFlight = sizeof(T) == 2 ? (kInter ? 2 : 1) : 4;
  extern __shared__ uint64_t turns[];   // [R / 2]
  __shared__ uint8_t s_named[kThreads + 1];   // per token of the CTA: a lower row names its position
  const long long item0 = static_cast<long long>(blockIdx.x) * kThreads, item = item0 + threadIdx.x;
  const bool live = item < p.items;
  const int per_token = p.units * p.chunks;
  const long long i = live ? item : 0;
  const long long token = i / per_token;
  const int rest = static_cast<int>(i - token * per_token);
  int c = rest / p.units;
  const int u = rest - c * p.units;
  const int b = static_cast<int>(token / p.n), s = static_cast<int>(token - static_cast<long long>(b) * p.n);
  int which = 0;
  while (c >= p.t[which].chunks) c -= p.t[which++].chunks;
  const AppendTensor& t = p.t[which];
  const bool turn_unit = u < p.turn_units;
  const bool turn = turn_unit && which < 2;
  constexpr int kHalf = kInter ? (N >= 2 ? N / 2 : 1) : N;   // pairs of a work item
  constexpr int kVecs = kInter && N >= 2 ? 1 : 2;            // vectors of a turning work item
  int col0, col1 = 0;
  if (turn_unit) {
    col0 = kInter ? u * (N >= 2 ? N : 2) : u * N;
    col1 = kInter ? col0 + 1 : col0 + p.R / 2;
  } else {
    col0 = p.R + (u - p.turn_units) * N;
  }
  // heads c, c + step, ...: the chunks' threads, neighbours in a warp, take neighbouring heads
  const int step = t.chunks;
  int n = live ? (t.heads - c + step - 1) / step : 0;
  const T* in = reinterpret_cast<const T*>(t.in) + b * t.in_b + s * t.in_l;
  using V = Vec<T, N>;
  V x[kHeadsInFlight][2];
  const auto load = [&](int i0) {
#pragma unroll
    for (int j = 0; j < kHeadsInFlight; ++j) {
      if (i0 + j >= n) break;
      const T* row = in + (c + (i0 + j) * step) * t.in_h;
      x[j][0] = *reinterpret_cast<const V*>(row + col0);
      if (kVecs == 2 && turn_unit) x[j][1] = *reinterpret_cast<const V*>(row + col1);
    }
  };
  griddep_wait();
  griddep_launch_dependents();
  // the first rows are on their way while the frequencies and the places are made ready
  const bool counted = p.count == nullptr || s < __ldg(p.count + b);
  if (!counted && t.pages != nullptr && t.out == nullptr) n = 0;   // padding
  load(0);
  int64_t at = p.pos != nullptr ? __ldg(p.pos + token) : static_cast<int64_t>(__ldg(p.start + b)) + s;
  const int64_t angle_at = p.rope_pos != nullptr && turn ? __ldg(p.rope_pos + token) : at;
  int64_t place = -1;   // row of the pages, of head 0
  if (t.pages != nullptr && counted && at >= 0 && at < (static_cast<int64_t>(p.M) << p.page_log2)) {
    const int entry = __ldg(p.table + static_cast<size_t>(b) * p.M + (at >> p.page_log2));
    if (entry >= 0 && entry < p.n_pages)
      place = ((static_cast<int64_t>(entry) * p.Hkv) << p.page_log2) + (at & ((1 << p.page_log2) - 1));
  }
  int bad = 0;   // some frequency is not finite
  for (int k = threadIdx.x; k < p.R / 2; k += kThreads) {
    const double radians = p.inv_freq[k];
    turns[k] = rope_turns(radians);
    bad |= not_finite(radians);
  }
  const long long token0 = item0 / per_token;
  if (p.pos != nullptr) {
    // a warp looks through the list for a token of the CTA at a time
    const long long last = min(item0 + kThreads, p.items) - 1;
    for (long long k = token0 + (threadIdx.x >> 5); k <= last / per_token; k += kThreads / 32) {
      const long long row0 = k / p.n * p.n;
      const int mine = __ldg(p.pos + k);
      bool hit = false;
      for (long long o = row0 + (threadIdx.x & 31); o < k; o += 32) hit |= __ldg(p.pos + o) == mine;
      hit = __any_sync(0xffffffffu, hit);
      if ((threadIdx.x & 31) == 0) s_named[k - token0] = hit ? 1 : 0;
    }
  }
  bad = __syncthreads_or(bad);
  if (p.pos != nullptr && live && s_named[token - token0] != 0) place = -1;
  float cs[kHalf], sn[kHalf];
  if (turn) {
#pragma unroll
    for (int k = 0; k < kHalf; ++k) {
      float si, co;
      rope_sincos(angle_at, turns[u * kHalf + k], &si, &co);
      cs[k] = co * p.mscale;
      sn[k] = si * p.mscale;
    }
    if (bad) {
#pragma unroll
      for (int k = 0; k < kHalf; ++k)
        if (not_finite(p.inv_freq[u * kHalf + k])) cs[k] = sn[k] = __uint_as_float(0x7fc00000u);
    }
  }
  T* const out = t.out == nullptr ? nullptr : reinterpret_cast<T*>(t.out) + (static_cast<size_t>(b) * t.heads * p.n + s) * p.D;
  for (int i0 = 0; i0 < n; i0 += kHeadsInFlight) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int j = 0; j < kHeadsInFlight; ++j) {
      if (i0 + j >= n) break;
      const int h = c + (i0 + j) * step;
      if constexpr (sizeof(T) == 2) {
        // pages and outputs are of one type: a vector is turned where it is
        if (turn) {
#pragma unroll
          for (int k = 0; k < kHalf; ++k) {
            T& xa = kVecs == 1 ? x[j][0].v[(2 * k) % N] : x[j][0].v[k % N];
            T& xb = kVecs == 1 ? x[j][0].v[(2 * k + 1) % N] : x[j][1].v[k % N];
            const float a = to_f(xa), d = to_f(xb);
            xa = from_f<T>(a * cs[k] - d * sn[k]);
            xb = from_f<T>(a * sn[k] + d * cs[k]);
          }
        }
        if (out != nullptr) {
          T* row = out + static_cast<size_t>(h) * p.n * p.D;
          *reinterpret_cast<V*>(row + col0) = x[j][0];
          if (kVecs == 2 && turn_unit) *reinterpret_cast<V*>(row + col1) = x[j][1];
        }
        if (place >= 0) {
          T* row = reinterpret_cast<T*>(t.pages) + (place + (static_cast<int64_t>(h) << p.page_log2)) * p.D;
          *reinterpret_cast<V*>(row + col0) = x[j][0];
          if (kVecs == 2 && turn_unit) *reinterpret_cast<V*>(row + col1) = x[j][1];
        }
      } else {
        if (turn) {
#pragma unroll
          for (int k = 0; k < kHalf; ++k) {
            T& xa = kVecs == 1 ? x[j][0].v[(2 * k) % N] : x[j][0].v[k % N];
            T& xb = kVecs == 1 ? x[j][0].v[(2 * k + 1) % N] : x[j][1].v[k % N];
            const float a = to_f(xa), d = to_f(xb);
            xa = from_f<T>(a * cs[k] - d * sn[k]);
            xb = from_f<T>(a * sn[k] + d * cs[k]);
          }
        }
#pragma unroll
        for (int w = 0; w < kVecs; ++w) {
          if (w == 1 && !turn_unit) break;
          const int col = w ? col1 : col0;
          if (out != nullptr) *reinterpret_cast<V*>(out + static_cast<size_t>(h) * p.n * p.D + col) = x[j][w];
          if (place >= 0) {
            Vec<bf16, N> r;
#pragma unroll
            for (int e = 0; e < N; ++e) r.v[e] = from_f<bf16>(to_f(x[j][w].v[e]));
            *reinterpret_cast<Vec<bf16, N>*>(t.pages + (place + (static_cast<int64_t>(h) << p.page_log2)) * p.D + col) = r;
          }
        }
      }
    }
  }
}

// Whether every row of the tensor starts on a vector of n elements of e bytes.
bool vectors_fit(const AppendTensor& t, int n, int e) {
  if (t.heads == 0) return true;
  const auto fits = [&](const void* p) { return reinterpret_cast<uintptr_t>(p) % (static_cast<size_t>(n) * e) == 0; };
  return fits(t.in) && fits(t.out) && t.in_b % n == 0 && t.in_h % n == 0 && t.in_l % n == 0;
}

}  // namespace

int launch_paged_append(const PagedAppendArgs& a, cudaStream_t stream) {
  AppendParams p{};
  const int64_t* st = a.strides;   // of k, v, q
  p.t[0] = AppendTensor{static_cast<const uint8_t*>(a.q), static_cast<uint8_t*>(a.q_out), nullptr, st[6], st[7], st[8], a.Hq, 0};
  p.t[1] = AppendTensor{static_cast<const uint8_t*>(a.k), static_cast<uint8_t*>(a.k_out), static_cast<bf16*>(a.k_pages), st[0], st[1], st[2], a.Hkv, 0};
  p.t[2] = AppendTensor{static_cast<const uint8_t*>(a.v), nullptr, static_cast<bf16*>(a.v_pages), st[3], st[4], st[5], a.Hkv, 0};
  p.inv_freq = a.inv_freq;
  p.table = a.table;
  p.start = a.start;
  p.count = a.count;
  p.pos = a.pos;
  p.rope_pos = a.rope_pos;
  p.n = a.n;
  p.D = a.D;
  p.R = a.R;
  p.M = a.M;
  p.n_pages = a.n_pages;
  p.Hkv = a.Hkv;
  while ((1 << p.page_log2) < a.page) ++p.page_log2;
  p.mscale = a.mscale;
  const int e = a.elem_bytes;
  int n = 16 / e;
  const bool wide = vectors_fit(p.t[0], n, e) && vectors_fit(p.t[1], n, e) && vectors_fit(p.t[2], n, e) &&
                    (a.interleaved ? a.R % n == 0 : (a.R / 2) % n == 0);
  if (!wide) n = 1;
  const int per_unit = a.interleaved ? (n >= 2 ? n / 2 : 1) : n;   // pairs of a work item
  p.turn_units = a.R / 2 / per_unit;
  p.units = p.turn_units + (a.D - a.R) / n;
  // Heads a thread walks over: see rope_kernel.cu.
  const long long tokens = static_cast<long long>(a.B) * a.n;
  const long long all = tokens * p.units * (a.Hq + 2LL * a.Hkv);
  const int chunk = static_cast<int>(std::min<long long>(8, std::max<long long>(1, all / (152 * 512))));
  for (AppendTensor& t : p.t) {
    t.chunks = (t.heads + chunk - 1) / chunk;
    p.chunks += t.chunks;
  }
  if (static_cast<long long>(p.chunks) * p.units > 0x7fffffffLL) return -2;
  p.items = tokens * p.chunks * p.units;
  const long long grid = (p.items + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffLL) return -2;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads), static_cast<size_t>(a.R / 2) * 8, stream, attr);
  cudaError_t r;
  if (e == 2)
    r = wide ? (a.interleaved ? cudaLaunchKernelEx(&cfg, paged_append_kernel<bf16, 8, true>, p)
                              : cudaLaunchKernelEx(&cfg, paged_append_kernel<bf16, 8, false>, p))
             : (a.interleaved ? cudaLaunchKernelEx(&cfg, paged_append_kernel<bf16, 1, true>, p)
                              : cudaLaunchKernelEx(&cfg, paged_append_kernel<bf16, 1, false>, p));
  else
    r = wide ? (a.interleaved ? cudaLaunchKernelEx(&cfg, paged_append_kernel<float, 4, true>, p)
                              : cudaLaunchKernelEx(&cfg, paged_append_kernel<float, 4, false>, p))
             : (a.interleaved ? cudaLaunchKernelEx(&cfg, paged_append_kernel<float, 1, true>, p)
                              : cudaLaunchKernelEx(&cfg, paged_append_kernel<float, 1, false>, p));
  return r == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
