// attn_prefix8.cu - two-view window attention over an 8-bit key/value memory.
//
// Query row r of head hq sits at memory position q0 + r and sees the keys lo <= j < hi of its row:
//   s_j = q . k_j / sqrt(d),  k_j = code * 2^(x - 127);  capped: s_j = c tanh(s_j / c)
//   o = sum_j softmax(s)_j v_j,  lse = ln sum_j e^{s_j}
// A seed row's own column, where it is among the row's keys, is the masked-input pair (k_i, v_i) instead
// (the leave-one-out view). A row that sees no key gives o = 0, lse = -inf; one that sees a key whose
// K or V row is NaN gives NaN.
//
// One warp per row, 32 keys at a time: a lane's key for the scores, four columns of a lane for the output.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "e4m3.cuh"
#include "kernels.cuh"
#include "ptx.cuh"
#include "route.cuh"

namespace cover {
namespace {

constexpr int kD = 128;
constexpr int kWarps = 8;

__global__ void __launch_bounds__(kWarps * 32) attn_prefix8_kernel(const Attn8Args a, long long rows) {
  __shared__ float s_q[kWarps][kD];
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kWarps + warp;   // of [B, Hq, Lq]
  if (row >= rows) return;
  const int r = static_cast<int>(row % a.Lq);
  const long long bh = row / a.Lq;
  const int hq = static_cast<int>(bh % a.Hq);
  const int b = static_cast<int>(bh / a.Hq);
  const int hkv = hq / (a.Hq / a.Hkv);
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + row * kD;
  for (int i = lane; i < kD; i += 32) s_q[warp][i] = __bfloat162float(q[i]);
  __syncwarp();
  const int pos = a.q0 + r;
  int slot = kNoSlot;
  for (int s = lane; s < a.n_seeds; s += 32)
    if (a.seed_idx[static_cast<size_t>(b) * a.n_seeds + s] == pos) slot = min(slot, s);
  slot = __reduce_min_sync(0xffffffffu, slot);
  const size_t lq = static_cast<size_t>(b) * a.Lq + r;
  const int lo = a.key_lo != nullptr ? max(0, a.key_lo[lq]) : 0;
  const int hi = a.key_hi != nullptr ? min(a.L, a.key_hi[lq]) : a.L;
  const size_t mem0 = (static_cast<size_t>(b) * a.Hkv + hkv) * a.L;
  const size_t self = (static_cast<size_t>(b) * a.Hkv + hkv) * a.n_seeds + (slot == kNoSlot ? 0 : slot);
  const uint8_t* k8 = static_cast<const uint8_t*>(a.k8);
  const uint8_t* v8 = static_cast<const uint8_t*>(a.v8);
  const float scale = 1.0f / sqrtf(static_cast<float>(kD));
  float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int j0 = lo; j0 < hi; j0 += 32) {
    const int j = j0 + lane;
    float s = -INFINITY;
    if (j < hi) {
      float dot = 0.0f;
      if (j == pos && slot != kNoSlot) {
        const __nv_bfloat16* ks = static_cast<const __nv_bfloat16*>(a.k_seedmask) + self * kD;
        for (int i = 0; i < kD; ++i) dot = fmaf(s_q[warp][i], __bfloat162float(ks[i]), dot);
      } else {
        const uint4* kr = reinterpret_cast<const uint4*>(k8 + (mem0 + j) * kD);
        for (int i = 0; i < kD / 16; ++i) {
          const uint4 c = __ldg(kr + i);
          const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 x = e4m3x2_values(w[e]), y = e4m3x2_values(w[e] >> 16);
            const float* qq = &s_q[warp][16 * i + 4 * e];
            dot = fmaf(qq[3], y.y, fmaf(qq[2], y.x, fmaf(qq[1], x.y, fmaf(qq[0], x.x, dot))));
          }
        }
        dot *= e4m3_scale(a.k_exp[mem0 + j]);
        if (a.v_exp[mem0 + j] == kExpNan) dot = e4m3_scale(kExpNan);
      }
      s = dot * scale;
      if (a.softcap > 0.0f) s = a.softcap * tanhf(s / a.softcap);
    }
    float top = s;
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float m_new = fmaxf(m, top);
    const float m_use = m_new == -INFINITY ? 0.0f : m_new;
    const float w = m == -INFINITY ? 0.0f : expf(m - m_use);
    const float p = expf(s - m_use);
    float sum = p;
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    l = l * w + sum;
    m = m_new;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= w;
    const int n = min(32, hi - j0);
    for (int t = 0; t < n; ++t) {
      const float pt = __shfl_sync(0xffffffffu, p, t);
      if (j0 + t == pos && slot != kNoSlot) {
        const __nv_bfloat16* vs = static_cast<const __nv_bfloat16*>(a.v_seedmask) + self * kD + 4 * lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(pt, __bfloat162float(vs[i]), o[i]);
      } else {
        const uint32_t c = __ldg(reinterpret_cast<const uint32_t*>(v8 + (mem0 + j0 + t) * kD) + lane);
        const float ps = pt * e4m3_scale(a.v_exp[mem0 + j0 + t]);
        const float2 x = e4m3x2_values(c), y = e4m3x2_values(c >> 16);
        o[0] = fmaf(ps, x.x, o[0]), o[1] = fmaf(ps, x.y, o[1]), o[2] = fmaf(ps, y.x, o[2]), o[3] = fmaf(ps, y.y, o[3]);
      }
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint2 r2 = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
  reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + row * kD)[lane] = r2;
  if (lane == 0 && a.lse != nullptr) a.lse[row] = m + logf(l);
}

}  // namespace

size_t attn_prefix8_workspace_bytes(int, int, int, int, int) { return 0; }

int launch_attn_prefix8(const Attn8Args& a, int*, cudaStream_t stream) {
  const long long rows = static_cast<long long>(a.B) * a.Hq * a.Lq;
  const long long grid = (rows + kWarps - 1) / kWarps;
  if (grid > 0x7fffffffLL) return -2;
  cudaLaunchAttribute attr[1];
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kWarps * 32), 0, stream, attr);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, attn_prefix8_kernel, a, rows);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
