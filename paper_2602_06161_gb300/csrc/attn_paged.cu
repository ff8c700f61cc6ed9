// attn_paged.cu - two-view window attention over a key/value memory in pages.
//
// k_pages, v_pages [n_pages, Hkv, page, 128] bf16; position t of sequence b is row t % page of the page table[b, t / page]. Query
// row r of head hq of sequence b sees the keys j of its sequence with key_lo <= j < key_hi, j < lens[b] and a page in the pool:
//   s_j = q . k_j / sqrt(d), capped: s_j = c tanh(s_j / c);  o = sum_j softmax(s)_j v_j,  lse = ln sum_j e^{s_j}
// A seed row's own column (its position is q0[b] + r), where it is among them, is the masked-input pair (k_i, v_i) instead. A row
// that sees no key gives o = 0, lse = -inf.
//
// One CTA a row, 128 keys at a time: a thread holds a key's score, then a column of the sum.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.cuh"
#include "ptx.cuh"
#include "route.cuh"

namespace cover {
namespace {

constexpr int kD = 128;

struct Params {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k_pages;
  const __nv_bfloat16* v_pages;
  const int32_t* table;
  const int32_t* lens;
  const __nv_bfloat16* k_seedmask;
  const __nv_bfloat16* v_seedmask;
  const int32_t* seed_idx;
  const int32_t* q0;
  const int32_t* key_lo;
  const int32_t* key_hi;
  __nv_bfloat16* out;
  float* lse;
  int n_pages, M, page_log2, n_seeds, Hq, Hkv, G, Lq;
  float scale, cap;
};

__global__ void __launch_bounds__(kD) attn_paged_row_kernel(const __grid_constant__ Params p) {
  __shared__ float s_q[kD], s_w[kD], s_red[4];
  __shared__ int64_t s_place[kD];   // element of the pages where the key's row starts, or -1
  __shared__ int s_slot;
  griddep_wait();
  griddep_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x;
  const int r = static_cast<int>(row % p.Lq), hq = static_cast<int>(row / p.Lq % p.Hq), b = static_cast<int>(row / p.Lq / p.Hq);
  const int h = hq / p.G;
  s_q[tid] = __bfloat162float(p.q[row * kD + tid]) * p.scale;
  if (tid == 0) s_slot = kNoSlot;
  __syncthreads();
  const long long i = static_cast<long long>(b) * p.Lq + r;
  const int64_t len = min(static_cast<int64_t>(__ldg(p.lens + b)), static_cast<int64_t>(p.M) << p.page_log2);
  const int64_t lo = max(0, p.key_lo != nullptr ? __ldg(p.key_lo + i) : 0);
  const int64_t hi = p.key_hi != nullptr ? min(len, static_cast<int64_t>(__ldg(p.key_hi + i))) : len;
  int64_t own = -1;
  if (p.n_seeds > 0) {
    own = static_cast<int64_t>(__ldg(p.q0 + b)) + r;
    for (int s = tid; s < p.n_seeds; s += kD)
      if (__ldg(p.seed_idx + static_cast<size_t>(b) * p.n_seeds + s) == own) atomicMin(&s_slot, s);
    __syncthreads();
    if (s_slot == kNoSlot) own = -1;
  }
  const size_t self = ((static_cast<size_t>(b) * p.Hkv + h) * p.n_seeds + (own >= 0 ? s_slot : 0)) * kD;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (int64_t j0 = lo; j0 < hi; j0 += kD) {
    const int64_t j = j0 + tid;
    int64_t place = -1;
    float s = -INFINITY;
    if (j < hi) {
      const int entry = __ldg(p.table + static_cast<size_t>(b) * p.M + (j >> p.page_log2));
      if (entry >= 0 && entry < p.n_pages)
        place = ((((static_cast<int64_t>(entry) * p.Hkv + h) << p.page_log2) + (j & ((1 << p.page_log2) - 1)))) * kD;
    }
    if (place >= 0) {
      const __nv_bfloat16* k = j == own ? p.k_seedmask + self : p.k_pages + place;
      s = 0.0f;
      for (int d = 0; d < kD; ++d) s = fmaf(s_q[d], __bfloat162float(k[d]), s);
      if (p.cap > 0.0f) s = p.cap * tanhf(s / p.cap);
    }
    s_place[tid] = place;
    float top = s;
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (lane == 0) s_red[warp] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    const float to = fmaxf(m, top), f = m == -INFINITY ? 0.0f : __expf(m - to);
    float w = s == -INFINITY ? 0.0f : __expf(s - to);
    s_w[tid] = w;
    for (int d = 16; d >= 1; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
    __syncthreads();
    if (lane == 0) s_red[warp] = w;
    __syncthreads();
    l = l * f + (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
    o *= f;
    m = to;
    for (int k = 0; k < kD && j0 + k < hi; ++k) {
      if (s_place[k] < 0) continue;
      const __nv_bfloat16* v = j0 + k == own ? p.v_seedmask + self : p.v_pages + s_place[k];
      o = fmaf(s_w[k], __bfloat162float(v[tid]), o);
    }
    __syncthreads();
  }
  p.out[row * kD + tid] = __float2bfloat16_rn(l == 0.0f ? 0.0f : o / l);
  if (tid == 0 && p.lse != nullptr) p.lse[row] = m + logf(l);
}

}  // namespace

size_t attn_paged_workspace_bytes(int, int, int, int, int, int) { return 0; }

int launch_attn_paged(const AttnPagedArgs& a, int*, cudaStream_t stream) {
  const long long rows = static_cast<long long>(a.B) * a.Hq * a.Lq;
  if (rows > 0x7fffffffLL) return -2;
  using bf16 = __nv_bfloat16;
  Params p{};
  p.q = static_cast<const bf16*>(a.q);
  p.k_pages = static_cast<const bf16*>(a.k_pages);
  p.v_pages = static_cast<const bf16*>(a.v_pages);
  p.table = a.table;
  p.lens = a.lens;
  p.k_seedmask = static_cast<const bf16*>(a.k_seedmask);
  p.v_seedmask = static_cast<const bf16*>(a.v_seedmask);
  p.seed_idx = a.seed_idx;
  p.q0 = a.q0;
  p.key_lo = a.key_lo;
  p.key_hi = a.key_hi;
  p.out = static_cast<bf16*>(a.out);
  p.lse = a.lse;
  p.n_pages = a.n_pages;
  p.M = a.M;
  while ((1 << p.page_log2) < a.page) ++p.page_log2;
  p.n_seeds = a.n_seeds;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.Lq = a.Lq;
  p.scale = 1.0f / sqrtf(static_cast<float>(kD));
  p.cap = a.softcap;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(rows)), dim3(kD), 0, stream, attr);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, attn_paged_row_kernel, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
