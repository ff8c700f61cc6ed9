// paged_append.cu - new rows of keys and values into a memory in pages, rotated to their positions on the way.
//
// k_pages, v_pages [n_pages, Hkv, page, D] bf16; position t of sequence b is row t % page of the page table[b, t / page].
// Row s of sequence b goes to start[b] + s (s < count[b]), or to pos[b, s], where of rows that name one position the
// lowest is taken; what has no page (a position outside the table, an entry outside the pool) is left out. k, and q beside
// it, turn by their positions first (the formulas and the angles of rope_kernel.cu), in fp32, and are rounded once.
//
// Bound by memory: every row is read and written once. A thread holds two 16-byte vector columns (R / 2 apart in the layout of halves; one of
// neighbouring pairs) of one token and walks over up to sixteen heads of q, k or v, so that its sines and cosines, and its token's place,
// serve all of them. Four heads are on their way at a time, into places of shared memory that are the thread's own: held in registers it
// was one head, and too few bytes were in flight. Threads are in the order (block of tokens, chunk of heads, token, column), so that a
// warp's threads walk over equally many heads.
// 4 x up to 8191 tokens, 32 + 8 + 8 heads of 128 (744 MB in bf16): 114 us, 6.5 TB/s; pairs of neighbours 124; fp32 rows 209, 6.6 TB/s. With a head
// held in registers 153, 176 and 232 us; 8 x 63 listed rows gain 0.1 of 4.2 us by that, 64 x 400 lose 16 of 51, so there is one form.
#include <cuda_bf16.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;
constexpr int kDepth = 4;   // heads of a thread in flight
constexpr int kMaxBlock = 8;   // tokens of a block
constexpr int kStageBytes = kDepth * 2 * kThreads * 16;
using bf16 = __nv_bfloat16;

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

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
  bool rest_pairs;          // the others take two vectors
  int block;                // tokens of a block
  int chunks;
  long long tokens, items;
  float mscale;
};

// T: element of the rows; N: elements of a thread's vector (16 bytes, or one element); kInter: pairs of neighbours.
template <typename T, int N, bool kInter>
__global__ void __launch_bounds__(kThreads, 4) paged_append_kernel(const __grid_constant__ AppendParams p) {
  extern __shared__ __align__(16) uint8_t smem[];   // wide rows: [kDepth][2][kThreads] vectors; turns [R / 2]
  constexpr bool kStaged = N > 1;
  uint64_t* const turns = reinterpret_cast<uint64_t*>(smem + (kStaged ? kStageBytes : 0));
  __shared__ uint8_t s_named[kThreads + 2 * kMaxBlock];   // per token of the CTA's blocks: a lower row names its position
  const long long item0 = static_cast<long long>(blockIdx.x) * kThreads, item = item0 + threadIdx.x;
  const bool live = item < p.items;
  const long long i = live ? item : 0, per_block = static_cast<long long>(p.units) * p.chunks * p.block;
  const long long block = i / per_block;
  const int in_block = static_cast<int>(i - block * per_block);
  const int per_chunk = p.units * static_cast<int>(min(static_cast<long long>(p.block), p.tokens - block * p.block));
  int c = in_block / per_chunk;
  const int in_chunk = in_block - c * per_chunk;
  const long long token = block * p.block + in_chunk / p.units;
  const int u = in_chunk % p.units;
  const int b = static_cast<int>(token / p.n), s = static_cast<int>(token - static_cast<long long>(b) * p.n);
  int which = 0;
  while (c >= p.t[which].chunks) c -= p.t[which++].chunks;
  const AppendTensor& t = p.t[which];
  const bool turn_unit = u < p.turn_units;
  const bool turn = turn_unit && which < 2;
  constexpr int kHalf = kInter ? (N >= 2 ? N / 2 : 1) : N;   // pairs of a work item
  constexpr int kVecs = kInter && N >= 2 ? 1 : 2;            // vectors of a turning work item
  int col0, col1 = 0;
  bool two = kVecs == 2;                                     // vectors of this one
  if (turn_unit) {
    col0 = kInter ? u * (N >= 2 ? N : 2) : u * N;
    col1 = kInter ? col0 + 1 : col0 + p.R / 2;
  } else {
    col0 = p.R + (u - p.turn_units) * N;
    col1 = col0 + (p.D - p.R) / 2;
    two = p.rest_pairs;
  }
  // heads c, c + step, ...: at the same turn the chunks of a block of tokens, which lie behind one another, take neighbouring heads
  const int step = t.chunks;
  int n = live ? (t.heads - c + step - 1) / step : 0;
  const T* in = reinterpret_cast<const T*>(t.in) + b * t.in_b + s * t.in_l;
  using V = Vec<T, N>;
  // a thread's places, in no other thread's way
  const auto slot_of = [&](int k, int w) { return smem + (((k % kDepth) * 2 + w) * kThreads + threadIdx.x) * 16; };
  // the k-th head's vectors, on their way to the thread's places
  const auto fetch = [&](int k) {
    if (k < n) {
      const T* row = in + (c + k * step) * t.in_h;
      copy_async16(smem_u32(slot_of(k, 0)), row + col0);
      if (two) copy_async16(smem_u32(slot_of(k, 1)), row + col1);
    }
    copy_async_commit();
  };
  griddep_wait();
  griddep_launch_dependents();
  // the first rows are on their way while the frequencies and the places are made ready
  const bool counted = p.count == nullptr || s < __ldg(p.count + b);
  if (!counted && t.pages != nullptr && t.out == nullptr) n = 0;   // padding
  if (kStaged) {
#pragma unroll
    for (int k = 0; k < kDepth; ++k) fetch(k);
  }
  const long long token0 = item0 / per_block * p.block;
  if (p.pos != nullptr) {
    // a warp looks through the lists for a token of the CTA's blocks at a time
    const long long last = (min(item0 + kThreads, p.items) - 1) / per_block;
    for (long long k = token0 + (threadIdx.x >> 5); k < min((last + 1) * p.block, p.tokens); k += kThreads / 32) {
      const long long row0 = k / p.n * p.n;
      const int mine = __ldg(p.pos + k);
      bool hit = false;
      for (long long o = row0 + (threadIdx.x & 31); o < k; o += 32) hit |= __ldg(p.pos + o) == mine;
      hit = __any_sync(0xffffffffu, hit);
      if ((threadIdx.x & 31) == 0) s_named[k - token0] = hit ? 1 : 0;
    }
  }
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
  for (int k = 0; k < n; ++k) {
    const int h = c + k * step;
    V x[2];
    if constexpr (kStaged) {
      copy_async_wait<kDepth - 1>();
      x[0] = *reinterpret_cast<const V*>(slot_of(k, 0));
      if (two) x[1] = *reinterpret_cast<const V*>(slot_of(k, 1));
    } else {
      const T* row = in + h * t.in_h;
      x[0] = *reinterpret_cast<const V*>(row + col0);
      if (two) x[1] = *reinterpret_cast<const V*>(row + col1);
    }
    if (turn) {
#pragma unroll
      for (int e = 0; e < kHalf; ++e) {
        T& xa = kVecs == 1 ? x[0].v[(2 * e) % N] : x[0].v[e % N];
        T& xb = kVecs == 1 ? x[0].v[(2 * e + 1) % N] : x[1].v[e % N];
        const float a = to_f(xa), d = to_f(xb);
        xa = from_f<T>(a * cs[e] - d * sn[e]);
        xb = from_f<T>(a * sn[e] + d * cs[e]);
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (w == 1 && !two) break;
      const int col = w ? col1 : col0;
      if (out != nullptr) *reinterpret_cast<V*>(out + static_cast<size_t>(h) * p.n * p.D + col) = x[w];
      if (place >= 0) {
        bf16* row = t.pages + (place + (static_cast<int64_t>(h) << p.page_log2)) * p.D + col;
        if constexpr (sizeof(T) == 2) {   // pages and rows are of one type
          *reinterpret_cast<V*>(row) = x[w];
        } else {
          Vec<bf16, N> r;
#pragma unroll
          for (int e = 0; e < N; ++e) r.v[e] = from_f<bf16>(to_f(x[w].v[e]));
          *reinterpret_cast<Vec<bf16, N>*>(row) = r;
        }
      }
    }
    if (kStaged) fetch(k + kDepth);   // (what was in its places has been stored)
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
  p.t[1] = AppendTensor{static_cast<const uint8_t*>(a.k), static_cast<uint8_t*>(a.k_out), static_cast<bf16*>(a.k_pages),
                        st[0], st[1], st[2], a.Hkv, 0};
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
  const int rest = (a.D - a.R) / n;   // vectors that do not turn
  p.rest_pairs = rest % 2 == 0;
  p.units = p.turn_units + (p.rest_pairs ? rest / 2 : rest);
  // Heads a thread walks over: as many, up to 16, as leave 512 threads an SM (10 x 1253 tokens, 32 + 32 + 32 heads of 64: 54 us with up to 8, 48 so).
  const long long tokens = static_cast<long long>(a.B) * a.n;
  const long long all = tokens * p.units * (a.Hq + 2LL * a.Hkv);
  const int chunk = static_cast<int>(std::min<long long>(16, std::max<long long>(1, all / (152 * 512))));
  for (AppendTensor& t : p.t) {
    t.chunks = (t.heads + chunk - 1) / chunk;
    p.chunks += t.chunks;
  }
  if (static_cast<long long>(p.chunks) * p.units > 0x7fffffffLL / kMaxBlock) return -2;
  // A CTA looks through a list for each of its blocks' tokens, so blocks are small where there is one (8 x 63 listed tokens, 64 heads of 64,
  // fp32: blocks of 8 5.1 us, of 2 4.4; 34 x 988 tokens in a run, 20 heads: 41 and 56).
  p.block = a.pos != nullptr ? 2 : kMaxBlock;
  p.tokens = tokens;
  p.items = tokens * p.chunks * p.units;
  const long long grid = (p.items + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffLL) return -2;
  cudaLaunchAttribute attr[1];
  const size_t smem = (wide ? kStageBytes : 0) + static_cast<size_t>(a.R / 2) * 8;
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, attr);
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
