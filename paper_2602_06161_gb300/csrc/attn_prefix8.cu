// attn_prefix8.cu - two-view window attention over an 8-bit key/value memory.
//
// Query row r of head hq sits at memory position q0 + r and sees the keys lo <= j < hi of its row:
//   s_j = q . k_j / sqrt(d),  k_j = code * 2^(x - 127);  capped: s_j = c tanh(s_j / c)
//   o = sum_j softmax(s)_j v_j,  lse = ln sum_j e^{s_j}
// A seed row's own column, where it is among the row's keys, is the masked-input pair (k_i, v_i) instead
// (the leave-one-out view). A row that sees no key gives o = 0, lse = -inf; one that sees a key whose
// K or V row is NaN gives NaN.
//
// The G = Hq / Hkv query heads of a KV head are packed: row p = g Lq + r of KV head (b, hkv) is query row r
// of head hkv G + g, and the packed rows are one run of the [B Hq Lq, D] view, cut into Q tiles of 128.
// A CTA takes one or two Q tiles against the KV tiles (128 keys) of one of nsplit parts of what its rows
// see. Codes arrive by bulk copies (64 rows are 8 KB in one piece); one warpgroup decodes K and one V to bf16
// (exact: a row's scale is a power of two) into the swizzled layout that the tensor cores read, and S = Q K^T, O += P V
// run as tcgen05.mma with S, P and O in tensor memory. Two softmax warpgroups keep one stream each:
//   shared Q (kPair = false): both streams are the same Q tile, on the even and the odd KV tiles, with sums and an
//     accumulator of their own that are merged at the end: the chain load - decode - S - softmax - P V of
//     one KV tile overlaps the next one's. For windows whose packed rows fill one Q tile.
//   pair (kPair = true): the streams are two Q tiles that read each decoded KV tile together.
// With nsplit > 1 the parts leave (m, l, O) in fp32 in the workspace and a second kernel combines them.
//
// Roles (640 threads): warps 0-3, 4-7 softmax of stream 0, 1 (thread = row); 8-11 decode K, 12-15 V; 16
// issues the products; 17 and 18 issue the copies of K and V.
// Shared memory: Q (32 or 64 KB) | rings of 8 KB entries of codes, K and V (4 or 2 each) | K, V in bf16 (2 x 32 KB each).
// Tensor memory: S0 | S1 (P overwrites their first 64 columns) | O0 | O1, 128 columns each.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "context.cuh"
#include "e4m3.cuh"
#include "kernels.cuh"
#include "ptx.cuh"
#include "route.cuh"
#include "tmap.cuh"

namespace cover {
namespace {

constexpr int kD = 128;
constexpr int kBM = 128;                   // rows per Q tile
constexpr int kBN = 128;                   // keys per KV tile
constexpr int kTileBytes = kBM * kD * 2;   // 32 KB
constexpr int kBoxBytes = kTileBytes / 2;  // one 64-column, 128-byte-swizzled box
constexpr int kHalf = kBN / 2;             // key rows of a ring entry
constexpr int kCodeBytes = kHalf * kD;     // 8 KB of codes
constexpr int kThreads = 640;
constexpr int kDecodeWarp = 8, kMmaWarp = 16, kLoadWarp = 17;
constexpr int kLaunchRegs = 96;            // registers per thread at launch (65536 / 640, rounded down to 8)
constexpr int kSoftmaxRegs = 160, kDecodeRegs = 56, kIssueRegs = 40;
static_assert(2 * 128 * kSoftmaxRegs + 2 * 128 * kDecodeRegs + 128 * kIssueRegs <= kThreads * kLaunchRegs, "register split");
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kSms = 152;                  // of this GPU; the split of the keys is chosen for it

struct Smem {
  uint8_t q_and_ring[3 * kTileBytes];   // Q | rings of K codes and of V codes
  uint8_t k[2][kTileBytes];
  uint8_t v[2][kTileBytes];
  uint64_t q_full;
  uint64_t c_full[2][4], c_empty[2][4]; // rings of K and V codes
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2], p_full[2];        // per stream
  uint64_t o_full, drain;
  uint32_t tmem_base;
  int abort;
  int lo, hi;                           // keys that some row of the CTA sees
  uint4 nan_keys[4];                    // per KV tile in turn: keys with a V row of NaN
  int slot[2 * kBM];                    // seed slot of a row's position, or kNoSlot
};
constexpr size_t kSmemBytes = sizeof(Smem) + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");

struct Params {
  const __nv_bfloat16* q;
  const uint8_t* k8;
  const uint8_t* v8;
  const uint8_t* k_exp;
  const uint8_t* v_exp;
  const __nv_bfloat16* k_seedmask;
  const __nv_bfloat16* v_seedmask;
  const int32_t* seed_idx;
  const int32_t* key_lo;
  const int32_t* key_hi;
  __nv_bfloat16* out;
  float* lse;
  float* part_o;     // [nsplit][rows][128]
  float2* part_ml;   // [nsplit][rows]
  int* status;
  long long rows;    // B * Hq * Lq
  int n_seeds, Hq, Hkv, G, Lq, Lk, q0, n_groups, nsplit;
  float scale_log2;  // log2(e) / sqrt(d)
  float cap_log2;    // cap * log2(e)
  float cap_in;      // 2 log2(e) / (cap sqrt(d))
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  const bool ok = mbar_wait(bar, parity, abort);
  return __all_sync(0xffffffffu, ok);
}

// All 256 threads of the two softmax warpgroups.
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

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

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Shared memory by its 32-bit address.
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// Bytes of x by the selector's nibbles; a nibble with its top bit set gives eight copies of that byte's sign.
template <uint32_t kSel>
__device__ __forceinline__ uint32_t prmt(uint32_t x) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(0), "n"(kSel));
  return d;
}

// A capped score in log2 units, c tanh(s / c) log2(e) = C (1 - 2 / (1 + e^{2 s / c})), C = c log2(e); the
// infinite and the vanishing exponential give the caps themselves.
__device__ __forceinline__ float capped(float s, float cap_in, float cap_log2) {
  const float t = ex2_approx(s * cap_in);
  return fmaf(-2.0f * cap_log2, rcp_approx(1.0f + t), cap_log2);
}

// Decodes half a row of codes: every other one of the eight 16-byte pieces of a row, into its row of a bf16 tile (two
// 64-column boxes, 16-byte chunks swizzled by row & 7). An e4m3 code's bits s eeee mmm, moved to s 0000eeee mmm0000, are
// the bf16 number code * 2^-120 (subnormal codes included), and one multiplication by m1 = 2^(120 + x - 127) gives the
// value; where that is above bf16's range, m1 = 2^120 and kTwo says to multiply by m2 = 2^(x - 127) too. Both are
// exact. The thread's pieces are u0 ^ 0, 2, 4, 6 with u0 the row's low bits (its partner's: u0 ^ 1), so that the reads
// and writes of eight lanes meet every bank. src: address of piece u0; d0, d1: of its first chunk, in its box and
// in the other one.
template <bool kTwo>
__device__ __forceinline__ void decode_half_row(uint32_t src, uint32_t d0, uint32_t d1, uint32_t m1, uint32_t m2) {
  uint4 next = lds128(src);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 c = next;
    if (i < 3) next = lds128(src ^ (32u * (i + 1)));
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t o[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // bytes 0, 1 (2, 3) sign-extended to 16 bits, moved up by four bits
      const uint32_t lo = (prmt<0x9180>(w[e]) << 4) & 0x87f087f0u;
      const uint32_t hi = (prmt<0xb3a2>(w[e]) << 4) & 0x87f087f0u;
      o[2 * e] = mul_bf16x2(lo, m1);
      o[2 * e + 1] = mul_bf16x2(hi, m1);
      if (kTwo) {
        o[2 * e] = mul_bf16x2(o[2 * e], m2);
        o[2 * e + 1] = mul_bf16x2(o[2 * e + 1], m2);
      }
    }
    const uint32_t d = (i & 2 ? d1 : d0) ^ (i & 1 ? 64u : 0u);
    sts128(d, o[0], o[1], o[2], o[3]);
    sts128(d ^ 16u, o[4], o[5], o[6], o[7]);
  }
}

__device__ __forceinline__ void decode(uint32_t src, uint32_t d0, uint32_t d1, int x, bool zero) {
  // bytes above 246 count as NaN (cover_kv8_write writes none but 255)
  const bool two = x > 134 && x <= kExpMax;
  uint32_t m1 = two ? 247u << 7 : static_cast<uint32_t>(x + 120) << 7;
  uint32_t m2 = two ? static_cast<uint32_t>(x) << 7 : 0x3f80u;
  if (x > kExpMax) m1 = 0x7fc0u;
  if (zero) m1 = 0;
  m1 |= m1 << 16;
  m2 |= m2 << 16;
  if (__any_sync(0xffffffffu, two)) decode_half_row<true>(src, d0, d1, m1, m2);
  else decode_half_row<false>(src, d0, d1, m1, m2);
}

// The exponent bytes of row lrow of four half tiles from half h on (zero from row `left` on).
struct FourBytes {
  uint32_t v[4];
  __device__ __forceinline__ void load(const uint8_t* exps, int h, int lrow, int left) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (h + i) * kHalf + lrow;
      v[i] = row < left ? __ldg(exps + row) : 0u;
    }
  }
  __device__ __forceinline__ uint32_t packed() const { return v[0] | (v[1] << 8) | (v[2] << 16) | (v[3] << 24); }
};

template <bool kPair, bool kCap>
__global__ void __launch_bounds__(kThreads, 1)
    attn_prefix8_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kQTiles = kPair ? 2 : 1;
  constexpr int kRing = kPair ? 2 : 4;   // entries of each ring
  uint8_t* const sm_q = sm.q_and_ring;
  uint8_t* const ring = sm.q_and_ring + kQTiles * kTileBytes;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // CTA (ks, group, hkv, b)
  const int ks = static_cast<int>(blockIdx.x) % p.nsplit;
  int rest = static_cast<int>(blockIdx.x) / p.nsplit;
  const int group = rest % p.n_groups;
  rest /= p.n_groups;
  const int hkv = rest % p.Hkv;
  const int b = rest / p.Hkv;
  const int n_packed = p.G * p.Lq;
  const int p0 = group * kQTiles * kBM;                                               // the CTA's first packed row
  const long long rowbase = (static_cast<long long>(b) * p.Hq + hkv * p.G) * p.Lq;    // packed row 0 in [B Hq Lq, D]
  const size_t mem0 = (static_cast<size_t>(b) * p.Hkv + hkv) * p.Lk;                  // the KV head's first memory row

  if (warp == kMmaWarp) {
    if (lane == 0) {
      mbar_init(&sm.q_full, 1);
      for (int i = 0; i < 4; ++i)
        for (int w = 0; w < 2; ++w) {
          mbar_init(&sm.c_full[w][i], 1);
          mbar_init(&sm.c_empty[w][i], 128);
        }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.k_full[i], 128);
        mbar_init(&sm.k_empty[i], 1);
        mbar_init(&sm.v_full[i], 128);
        mbar_init(&sm.v_empty[i], 1);
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], kBM);
      }
      mbar_init(&sm.o_full, 1);
      mbar_init(&sm.drain, 1);
      sm.abort = 0;
      sm.lo = 0x7fffffff;
      sm.hi = 0;
      fence_mbar_init();
      tma_prefetch_desc(&tm_q);
    }
    __syncwarp();
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  if (p.n_seeds > 0 && tid < 2 * kBM) sm.slot[tid] = kNoSlot;
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = sm.tmem_base;
  griddep_wait();
  griddep_launch_dependents();

  // ---------------- the rows' keys ----------------
  // softmax thread: its row, the keys [row_lo, row_hi) that it sees
  const int stream = warp >> 2;                       // of a softmax warp
  const int R = tid & (kBM - 1);
  const int P = p0 + (kPair ? stream * kBM : 0) + R;
  const bool valid = warp < kDecodeWarp && P < n_packed;
  const int r = valid ? P % p.Lq : 0;
  int row_lo = 0, row_hi = p.Lk;
  if (valid && p.key_lo != nullptr) row_lo = max(0, __ldg(p.key_lo + static_cast<size_t>(b) * p.Lq + r));
  if (valid && p.key_hi != nullptr) row_hi = min(p.Lk, __ldg(p.key_hi + static_cast<size_t>(b) * p.Lq + r));
  int t0 = 0, t1 = (p.Lk + kBN - 1) / kBN;            // KV tiles of which some row sees a key
  if (p.key_lo != nullptr || p.key_hi != nullptr) {
    if (warp < kDecodeWarp) {
      const bool some = valid && row_lo < row_hi;
      const int lo = __reduce_min_sync(0xffffffffu, some ? row_lo : 0x7fffffff);
      const int hi = __reduce_max_sync(0xffffffffu, some ? row_hi : 0);
      if (lane == 0 && hi > 0) {
        atomicMin(&sm.lo, lo);
        atomicMax(&sm.hi, hi);
      }
    }
    __syncthreads();
    const int lo = sm.lo, hi = sm.hi;
    t0 = hi > 0 ? lo / kBN : 0;
    t1 = hi > 0 ? (hi + kBN - 1) / kBN : 0;
  }
  // this part's KV tiles: j0 .. j0 + nt - 1
  const int each = (t1 - t0) / p.nsplit, more = (t1 - t0) % p.nsplit;
  const int j0 = t0 + ks * each + min(ks, more);
  const int nt = each + (ks < more ? 1 : 0);
  const bool two_tiles = kPair && p0 + kBM < n_packed;   // the pair's second Q tile has rows

  if (warp >= kMmaWarp) {
    setmaxnreg_dec<kIssueRegs>();
    const int which = warp - kLoadWarp;   // 0: K (and Q), 1: V
    if ((which == 0 || which == 1) && lane == 0 && nt > 0) {
      // ---------------- copies ----------------
      if (which == 0) {
        mbar_arrive_expect_tx(&sm.q_full, kQTiles * kTileBytes);
        for (int t = 0; t < kQTiles; ++t)
          for (int h = 0; h < 2; ++h)
            tma_load_4d(sm_q + t * kTileBytes + h * kBoxBytes, &tm_q, &sm.q_full, 64 * h,
                        static_cast<int>(rowbase) + p0 + t * kBM, 0, 0);
      }
      const uint8_t* src = (which ? p.v8 : p.k8) + mem0 * kD;
      uint8_t* const dst = ring + which * kRing * kCodeBytes;
      // half tiles with a key of the memory
      const int halves = min(2 * nt, (p.Lk - j0 * kBN + kHalf - 1) / kHalf);
      int e = 0;
      bool ok = true;
      for (; e < halves; ++e) {
        const int st = e % kRing;
        if (e >= kRing) ok = mbar_wait(&sm.c_empty[which][st], (e / kRing - 1) & 1, &sm.abort);
        if (!ok) break;
        const int key0 = j0 * kBN + e * kHalf;
        const uint32_t bytes = static_cast<uint32_t>(min(kHalf, p.Lk - key0)) * kD;
        mbar_arrive_expect_tx(&sm.c_full[which][st], bytes);
        bulk_load(smem_u32(dst + st * kCodeBytes), src + static_cast<size_t>(key0) * kD, bytes, &sm.c_full[which][st]);
      }
      if (!ok) {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 70);
        sm.abort = 1;
      }
      // every copy lands before the CTA's shared memory is released, whatever the other roles did
      if (which == 0) mbar_wait(&sm.q_full, 0, nullptr);
      for (int f = max(0, e - kRing); f < e; ++f) mbar_wait(&sm.c_full[which][f % kRing], (f / kRing) & 1, nullptr);
    } else if (warp == kMmaWarp && lane == 0 && nt > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_qk = idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t id_pv = idesc_bf16_f32(kBM, kD, false, true);
      constexpr uint64_t kTileDesc = kTileBytes >> 4;
      const uint64_t dq = sdesc_sw128(smem_u32(sm_q), 16, 1024);
      const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
      const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), kBoxBytes, 1024);
      // S[s] = Q . K(stage)^T
      auto issue_s = [&](int s, int st) {
        uint64_t a = dq + (kPair ? s * kTileDesc : 0), kb = dk + st * kTileDesc;
        asm volatile("" : "+l"(a), "+l"(kb));   // descriptors are added up here, not kept in registers
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          const uint64_t off = static_cast<uint64_t>(((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4);
          umma_ss(tbase + s * kBN, a + off, kb + off, id_qk, kk > 0 ? 1u : 0u);
        }
        umma_commit(&sm.s_full[s]);
      };
      // O[s] (+)= P[s] . V(stage)
      auto issue_pv = [&](int s, int st, bool acc) {
        uint64_t vb = dv + st * kTileDesc;
        asm volatile("" : "+l"(vb));
#pragma unroll
        for (int kk = 0; kk < kBN / 16; ++kk)
          umma_ts(tbase + 2 * kBN + s * kD, tbase + s * kBN + 8 * kk,
                  vb + static_cast<uint64_t>((kk * 2048) >> 4), id_pv, (acc || kk > 0) ? 1u : 0u);
      };
      auto wait = [&](uint64_t* bar, int phase) {
        const bool ok = mbar_wait(bar, phase & 1, &sm.abort);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      bool ok = wait(&sm.q_full, 0);
      if (kPair) {
        if (ok && (ok = wait(&sm.k_full[0], 0))) {
          issue_s(0, 0);
          if (two_tiles) issue_s(1, 0);
          umma_commit(&sm.k_empty[0]);
        }
        for (int j = 0; j < nt && ok; ++j) {
          const int st = j & 1;
          const bool next = j + 1 < nt;
          ok = wait(&sm.p_full[0], j) && wait(&sm.v_full[st], j >> 1);
          if (!ok) break;
          issue_pv(0, st, j > 0);
          if (next) {
            ok = wait(&sm.k_full[st ^ 1], (j + 1) >> 1);
            if (!ok) break;
            issue_s(0, st ^ 1);
          }
          if (two_tiles) {
            ok = wait(&sm.p_full[1], j);
            if (!ok) break;
            issue_pv(1, st, j > 0);
            if (next) issue_s(1, st ^ 1);
          }
          umma_commit(&sm.v_empty[st]);
          if (next) umma_commit(&sm.k_empty[st ^ 1]);
        }
      } else {
        // stream j & 1 takes tile j, from stage j & 1
        for (int j = 0; j < 2 && j < nt && ok; ++j) {
          ok = wait(&sm.k_full[j], 0);
          if (!ok) break;
          issue_s(j, j);
          umma_commit(&sm.k_empty[j]);
        }
        for (int j = 0; j < nt && ok; ++j) {
          const int s = j & 1;
          ok = wait(&sm.p_full[s], j >> 1) && wait(&sm.v_full[s], j >> 1);
          if (!ok) break;
          issue_pv(s, s, j > 1);
          umma_commit(&sm.v_empty[s]);
          if (j + 2 < nt) {
            ok = wait(&sm.k_full[s], (j + 2) >> 1);
            if (!ok) break;
            issue_s(s, s);
            umma_commit(&sm.k_empty[s]);
          }
        }
      }
      if (ok) {
        umma_commit(&sm.o_full);
      } else {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 71);
        sm.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&sm.drain);
      mbar_wait(&sm.drain, 0, nullptr);
    }
    __syncwarp();
  } else if (warp >= kDecodeWarp) {
    // ---------------- decoding ----------------
    setmaxnreg_dec<kDecodeRegs>();
    const int which = (warp - kDecodeWarp) >> 2;   // 0: K, 1: V
    const int t = tid & 127;
    const int lrow = t & (kHalf - 1);              // two threads a row of a half tile
    const uint32_t u0 = static_cast<uint32_t>((lrow ^ (t >> 6)) & 7);
    const uint32_t codes = smem_u32(ring + which * kRing * kCodeBytes + lrow * kD) + u0 * 16;
    const uint32_t tile = smem_u32(which ? sm.v[0] : sm.k[0]) + lrow * 128 + (((u0 & 3) << 5) ^ ((lrow & 7) << 4));
    const uint32_t box = (u0 >> 2) * kBoxBytes;
    const int first = j0 * kBN;                    // this part's first key
    const int left = min(p.Lk - first, nt * kBN);  // keys of this part
    // exponent bytes are fetched four half tiles at a time, four to eight ahead of their use
    const uint8_t* exps = (which ? p.v_exp : p.k_exp) + mem0 + first;
    const uint8_t* v_exps = p.v_exp + mem0 + first;
    FourBytes x_next, v_next;
    x_next.load(exps, 0, lrow, left);
    v_next.load(v_exps, 0, lrow, left);
    uint32_t xs = 0, vs = 0;
    bool ok = true;
    for (int h = 0; h < 2 * nt; ++h) {   // half h & 1 of tile h / 2
      const int j = h >> 1, st = j & 1;
      if ((h & 3) == 0) {
        xs = x_next.packed();
        x_next.load(exps, h + 4, lrow, left);
        if (which == 0) {
          vs = v_next.packed();
          v_next.load(v_exps, h + 4, lrow, left);
        }
      }
      const bool zero = h * kHalf + lrow >= left;
      const int x = (xs >> (8 * (h & 3))) & 255, xv = which ? x : static_cast<int>((vs >> (8 * (h & 3))) & 255);
      const bool v_nan = xv > kExpMax;
      const uint32_t nans = __ballot_sync(0xffffffffu, v_nan);
      if ((h & 1) == 0 && j >= 2) ok = warp_wait(which ? &sm.v_empty[st] : &sm.k_empty[st], ((j >> 1) - 1) & 1, &sm.abort);
      const bool copied = h * kHalf < left;        // a half past the memory is not copied
      ok = ok && (!copied || warp_wait(&sm.c_full[which][h % kRing], (h / kRing) & 1, &sm.abort));
      if (!ok) break;
      // tile j - 4 has passed its softmax: S of tile j - 2 came after it
      if (which == 0 && t < kHalf && lane == 0)
        reinterpret_cast<uint32_t*>(&sm.nan_keys[j & 3])[2 * (h & 1) + (t >> 5)] = nans;
      // a weight of zero times NaN is NaN: V rows of NaN are decoded as zeros, and the scores of their
      // keys are made NaN instead
      const uint32_t to = tile + st * kTileBytes + (h & 1) * kHalf * 128;
      decode(codes + (h % kRing) * kCodeBytes, to + box, to + (kBoxBytes - box), x, zero || (which && v_nan));
      if (copied) mbar_arrive(&sm.c_empty[which][h % kRing]);
      if (h & 1) {
        fence_proxy_async_smem();
        mbar_arrive(which ? &sm.v_full[st] : &sm.k_full[st]);
      }
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 72);
      sm.abort = 1;
    }
  } else {
    // ---------------- softmax ----------------
    setmaxnreg_inc<kSoftmaxRegs>();
    int slot = kNoSlot;
    if (p.n_seeds > 0) {
      // the CTA's rows stand at up to 256 positions: r itself, or r - r0 around Lq
      const int r0 = p.Lq <= 2 * kBM ? 0 : p0 % p.Lq;
      const int32_t* seeds = p.seed_idx + static_cast<size_t>(b) * p.n_seeds;
      for (int s = tid; s < p.n_seeds; s += 2 * kBM) {
        const int at = __ldg(seeds + s) - p.q0;
        if (at < 0 || at >= p.Lq) continue;
        const int i = at >= r0 ? at - r0 : at - r0 + p.Lq;
        if (i < 2 * kBM) atomicMin(&sm.slot[i], s);
      }
      softmax_sync();
      if (valid) slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq];
    }
    const int pos = p.q0 + r;
    const bool is_seed = slot != kNoSlot;
    const bool warp_seed = __any_sync(0xffffffffu, is_seed);
    const size_t self = (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds + (is_seed ? slot : 0);
    // the seed rows' own scores (log2 units), in the first part alone
    float s_self = -INFINITY;
    if (ks == 0 && is_seed && pos >= row_lo && pos < row_hi) {
      const uint4* qr = reinterpret_cast<const uint4*>(p.q + (rowbase + P) * kD);
      const uint4* kr = reinterpret_cast<const uint4*>(p.k_seedmask + self * kD);
      float d0 = 0.0f, d1 = 0.0f;
#pragma unroll 4
      for (int i = 0; i < kD / 8; ++i) {
        const uint4 a = __ldg(qr + i), c = __ldg(kr + i);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          d0 = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), d0);
          d1 = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), d1);
        }
      }
      s_self = kCap ? capped(d0 + d1, p.cap_in, p.cap_log2) : (d0 + d1) * p.scale_log2;
    }
    const bool warp_live = __any_sync(0xffffffffu, valid);
    const uint32_t s_addr = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16) + stream * kBN;
    const uint32_t o_addr = s_addr + 2 * kBN;
    const float scale = kCap ? 1.0f : p.scale_log2;
    const int jstep = kPair ? 1 : 2;
    float m_run = -INFINITY, l_run = 0.0f;
    bool ok = true;
    const int jend = kPair && stream == 1 && !two_tiles ? 0 : nt;
    int i = 0;   // the stream's step
    for (int j = kPair ? 0 : stream; j < jend; j += jstep, ++i) {
      ok = warp_wait(&sm.s_full[stream], i & 1, &sm.abort);
      if (!ok) break;
      tc_fence_after_sync();
      const int key0 = (j0 + j) * kBN;
      const int cl = row_lo - key0, ch = row_hi - key0;   // columns cl <= c < ch are seen
      if (!__any_sync(0xffffffffu, valid && max(cl, 0) < min(ch, kBN))) {
        // no row of the warp sees a key here; rows without a query row are never read
        if (warp_live) {
          const uint32_t zeros[32] = {};
          tmem_st32(s_addr, zeros);
          tmem_st32(s_addr + 32, zeros);
          tmem_st_wait();
        }
        tc_fence_before_sync();
        mbar_arrive(&sm.p_full[stream]);
        continue;
      }
      uint32_t raw[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, raw[c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_wait(raw[c]);
      float* s = reinterpret_cast<float*>(&raw[0][0]);
      if (kCap) {
#pragma unroll
        for (int c = 0; c < kBN; ++c) s[c] = capped(s[c], p.cap_in, p.cap_log2);
      }
      const uint4 nan4 = sm.nan_keys[j & 3];
      if ((nan4.x | nan4.y | nan4.z | nan4.w) != 0) {
        const uint32_t nw[4] = {nan4.x, nan4.y, nan4.z, nan4.w};
#pragma unroll
        for (int c = 0; c < kBN; ++c)
          if ((nw[c >> 5] >> (c & 31)) & 1u) s[c] = __uint_as_float(0x7fc00000u);
      }
      if (__any_sync(0xffffffffu, valid && (cl > 0 || ch < kBN))) {
#pragma unroll
        for (int c = 0; c < kBN; ++c)
          if (c < cl || c >= ch) s[c] = -INFINITY;
      }
      if (warp_seed && __any_sync(0xffffffffu, is_seed && pos >= key0 && pos < key0 + kBN)) {
        // a seed row does not see its own cached column
        const int dc = is_seed ? pos - key0 : -1;
#pragma unroll
        for (int c = 0; c < kBN; ++c)
          if (c == dc) s[c] = -INFINITY;
      }
      // row maximum: four independent 3-input max chains
      float mx0 = s[0], mx1 = s[1], mx2 = s[2], mx3 = s[3];
#pragma unroll
      for (int c = 4; c + 8 <= kBN; c += 8) {
        mx0 = fmax3(mx0, s[c], s[c + 1]);
        mx1 = fmax3(mx1, s[c + 2], s[c + 3]);
        mx2 = fmax3(mx2, s[c + 4], s[c + 5]);
        mx3 = fmax3(mx3, s[c + 6], s[c + 7]);
      }
      mx0 = fmax3(mx0, s[kBN - 4], s[kBN - 3]);
      mx1 = fmax3(mx1, s[kBN - 2], s[kBN - 1]);
      const float m_tile = fmax3(mx0, mx1, fmaxf(mx2, mx3)) * scale;
      float alpha = 1.0f;
      bool rescaled = false;
      if (m_tile > m_run + kRescaleThreshold) {
        alpha = (m_run == -INFINITY) ? 0.0f : ex2_approx(m_run - m_tile);
        m_run = m_tile;
        rescaled = true;
      }
      const float m_use = (m_run == -INFINITY) ? 0.0f : m_run;
      // p = 2^(s * scale - m) on pairs; four independent partial row sums
      const uint64_t scale2 = f2_pack(scale, scale);
      const uint64_t negm2 = f2_pack(-m_use, -m_use);
      uint64_t acc2[4] = {0, 0, 0, 0};
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint32_t packed[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          float x0, x1;
          f2_unpack(f2_fma(f2_pack(s[64 * hf + 2 * c], s[64 * hf + 2 * c + 1]), scale2, negm2), x0, x1);
          const float e0 = ex2_approx(x0);
          const float e1 = ex2_approx(x1);
          packed[c] = pack_bf16x2(e0, e1);
          acc2[c & 3] = f2_add(acc2[c & 3], f2_pack(e0, e1));
        }
        tmem_st32(s_addr + 32 * hf, packed);
      }
      float rs[4];
      f2_unpack(f2_add(acc2[0], acc2[1]), rs[0], rs[1]);
      f2_unpack(f2_add(acc2[2], acc2[3]), rs[2], rs[3]);
      l_run = l_run * alpha + ((rs[0] + rs[1]) + (rs[2] + rs[3]));
      if (i > 0 && __any_sync(0xffffffffu, rescaled)) {
        // O holds the stream's earlier products (complete: the commit of this S came after them)
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t o[32];
          tmem_ld32(o_addr + 32 * c, o);
          tmem_ld_wait(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
          tmem_st32(o_addr + 32 * c, o);
        }
      }
      tmem_st_wait();
      tc_fence_before_sync();
      mbar_arrive(&sm.p_full[stream]);
    }
    if (ok && nt > 0) ok = warp_wait(&sm.o_full, 0, &sm.abort);
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 73);
      sm.abort = 1;
    }

    // ---------------- the rows' results ----------------
    // of the thread's row: the sums of the streams that worked on it, and the accumulators' weights
    tc_fence_after_sync();
    float m = m_run, l = l_run, w[2] = {1.0f, 1.0f};
    const uint32_t o0 = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 2 * kBN;
    int c0 = 0, c1 = 4;   // 32-column chunks that this thread finishes
    if (!kPair) {
      float2* ml = reinterpret_cast<float2*>(sm_q);   // every product is complete: Q is not read any more
      if (ok) ml[stream * kBM + R] = make_float2(m_run, l_run);
      softmax_sync();
      const float2 a = ml[R], c = ml[kBM + R];
      m = fmaxf(a.x, c.x);
      const float m_use = m == -INFINITY ? 0.0f : m;
      w[0] = a.x == -INFINITY ? 0.0f : ex2_approx(a.x - m_use);
      w[1] = c.x == -INFINITY ? 0.0f : ex2_approx(c.x - m_use);
      l = w[0] * a.y + w[1] * c.y;
      c0 = 2 * stream, c1 = c0 + 2;
    }
    const float m_all = fmaxf(m, s_self);
    float p_self = 0.0f;
    if (s_self != -INFINITY) {
      const float f = m == -INFINITY ? 0.0f : ex2_approx(m - m_all);
      p_self = ex2_approx(s_self - m_all);
      l = l * f + p_self;
      w[0] *= f, w[1] *= f;
      m = m_all;
    }
    if (s_self != s_self) l = s_self;   // NaN in the masked-input pair
    const bool self_here = __any_sync(0xffffffffu, p_self != 0.0f);
    const long long orow = rowbase + P;
    const bool split = p.nsplit > 1;
    // 1 / l, once a row; zero where no key was seen
    const float inv = split ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
    if (ok && warp_live) {
#pragma unroll 1
      for (int c = c0; c < c1; ++c) {
        float o[32];
        if (nt > 0) {
          uint32_t x[32];
          tmem_ld32((kPair ? o_addr : o0) + 32 * c, x);
          tmem_ld_wait(x);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = w[0] == 0.0f ? 0.0f : __uint_as_float(x[e]) * w[0];
          if (!kPair && nt > 1) {
            tmem_ld32(o0 + kD + 32 * c, x);
            tmem_ld_wait(x);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(x[e]), w[1], o[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.0f;
        }
        if (self_here && p_self != 0.0f) {
          const uint4* vr = reinterpret_cast<const uint4*>(p.v_seedmask + self * kD + 32 * c);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint4 a = __ldg(vr + e);
            const uint32_t x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              o[8 * e + 2 * f] = fmaf(p_self, __uint_as_float(x[f] << 16), o[8 * e + 2 * f]);
              o[8 * e + 2 * f + 1] = fmaf(p_self, __uint_as_float(x[f] & 0xffff0000u), o[8 * e + 2 * f + 1]);
            }
          }
        }
        if (valid && split) {
          float4* dst = reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(ks) * p.rows + orow) * kD + 32 * c);
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        } else if (valid) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + orow * kD + 32 * c);
          // a NaN sum makes the whole row NaN
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                                pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
        }
        __syncwarp();   // the next chunk is loaded by the whole warp
      }
      if (valid && c0 == 0) {
        if (split) p.part_ml[static_cast<size_t>(ks) * p.rows + orow] = make_float2(m, l);
        else if (p.lse != nullptr) p.lse[orow] = (m + lg2_approx(l)) * 0.6931471805599453f;
      }
    }
    tc_fence_before_sync();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, 512);
  }
}

// Combines the parts of every row: one warp a row, four columns a lane.
constexpr int kCombineWarps = 4;
__global__ void __launch_bounds__(kCombineWarps * 32)
    attn_prefix8_combine_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, int nsplit,
                                long long rows, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5);
  if (row >= rows) return;
  float m = -INFINITY;
  for (int j = lane; j < nsplit; j += 32) m = fmaxf(m, part_ml[j * rows + row].x);
  for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  const float m_use = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int j = 0; j < nsplit; ++j) {
    const float2 ml = part_ml[j * rows + row];
    const float4 o = *reinterpret_cast<const float4*>(part_o + (j * rows + row) * kD + 4 * lane);
    const float w = ml.x == -INFINITY ? 0.0f : ex2_approx(ml.x - m_use);
    l = fmaf(w, ml.y, l);
    // parts that saw no key hold zeros; what rounds a weight to zero adds nothing
    acc.x = fmaf(w, o.x, acc.x);
    acc.y = fmaf(w, o.y, acc.y);
    acc.z = fmaf(w, o.z, acc.z);
    acc.w = fmaf(w, o.w, acc.w);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  reinterpret_cast<uint2*>(out + row * kD)[lane] =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (lane == 0 && lse != nullptr) lse[row] = (m + lg2_approx(l)) * 0.6931471805599453f;
}

struct Plan {
  bool pair;
  int n_groups, nsplit;
};

// One Q tile or two of a KV head a CTA, and the parts of the keys.
Plan plan_of(int B, int Hq, int Hkv, int Lq, int L) {
  Plan best{};
  double best_us = 0.0;
  const int G = Hq / Hkv;
  const long long n_qt = (static_cast<long long>(G) * Lq + kBM - 1) / kBM;
  const int nkv = (L + kBN - 1) / kBN;
  for (int pair = 0; pair < 2; ++pair) {
    if (pair && n_qt < 2) continue;
    const long long groups = pair ? (n_qt + 1) / 2 : n_qt;
    const long long units = groups * Hkv * B;
    for (int ns = 1; ns <= nkv && ns <= 64; ++ns) {
      const long long waves = (units * ns + kSms - 1) / kSms;
      const int tiles = (nkv + ns - 1) / ns;
      const double us = waves * (3.0 + (pair ? 1.3 : 0.75) * tiles) + (ns > 1 ? 1.5 + 0.0000003 * ns * units * (pair ? 256 : 128) * 528 / 4 : 0.0);
      if (best.nsplit == 0 || us < best_us) {
        best = Plan{pair != 0, static_cast<int>(groups), ns};
        best_us = us;
      }
      if (units * ns > 8 * kSms) break;
    }
  }
  return best;
}

size_t part_bytes(long long rows, int nsplit) {
  return nsplit <= 1 ? 0 : static_cast<size_t>(rows) * nsplit * (kD * sizeof(float) + sizeof(float2));
}

}  // namespace

size_t attn_prefix8_workspace_bytes(int B, int Hq, int Hkv, int Lq, int L) {
  return part_bytes(static_cast<long long>(B) * Hq * Lq, plan_of(B, Hq, Hkv, Lq, L).nsplit);
}

int launch_attn_prefix8(const Attn8Args& a, int* status, cudaStream_t stream) {
  const long long rows = static_cast<long long>(a.B) * a.Hq * a.Lq;
  if (rows + 2 * kBM > 0x7fffffffLL) return -2;
  const Plan plan = plan_of(a.B, a.Hq, a.Hkv, a.Lq, a.L);
  const long long grid = static_cast<long long>(plan.n_groups) * a.Hkv * a.B * plan.nsplit;
  if (grid > 0x7fffffffLL) return -2;
  static ContextCache<int> setup;
  int unused = 0;
  const int rc = setup.get(&unused, [&](int&) {
    for (auto fn : {attn_prefix8_kernel<false, false>, attn_prefix8_kernel<false, true>, attn_prefix8_kernel<true, false>,
                    attn_prefix8_kernel<true, true>}) {
      if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes)) != cudaSuccess)
        return -3;
      // the register split inside the kernel assumes exactly kLaunchRegs per thread at launch; any
      // other count could leave setmaxnreg.inc waiting, so refuse to launch
      cudaFuncAttributes fa;
      if (cudaFuncGetAttributes(&fa, fn) != cudaSuccess || fa.numRegs != kLaunchRegs) return -2;
    }
    return 0;
  });
  if (rc != 0) return rc;
  CUtensorMap tq;
  if (!make_bf16_map_4d(&tq, a.q, kD, static_cast<uint64_t>(rows), 1, 1, kBM)) return -3;
  const float log2e = 1.4426950408889634f, root = sqrtf(static_cast<float>(kD));
  Params p{};
  p.q = static_cast<const __nv_bfloat16*>(a.q);
  p.k8 = static_cast<const uint8_t*>(a.k8);
  p.v8 = static_cast<const uint8_t*>(a.v8);
  p.k_exp = a.k_exp;
  p.v_exp = a.v_exp;
  p.k_seedmask = static_cast<const __nv_bfloat16*>(a.k_seedmask);
  p.v_seedmask = static_cast<const __nv_bfloat16*>(a.v_seedmask);
  p.seed_idx = a.seed_idx;
  p.key_lo = a.key_lo;
  p.key_hi = a.key_hi;
  p.out = static_cast<__nv_bfloat16*>(a.out);
  p.lse = a.lse;
  p.part_o = static_cast<float*>(a.workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + static_cast<size_t>(rows) * plan.nsplit * kD);
  p.status = status;
  p.rows = rows;
  p.n_seeds = a.n_seeds;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.Lq = a.Lq;
  p.Lk = a.L;
  p.q0 = a.q0;
  p.n_groups = plan.n_groups;
  p.nsplit = plan.nsplit;
  p.scale_log2 = log2e / root;
  const bool cap = a.softcap > 0.0f;
  p.cap_log2 = a.softcap * log2e;
  p.cap_in = cap ? 2.0f * log2e / (a.softcap * root) : 0.0f;
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads), kSmemBytes, stream, attr);
  auto kernel = plan.pair ? (cap ? attn_prefix8_kernel<true, true> : attn_prefix8_kernel<true, false>)
                          : (cap ? attn_prefix8_kernel<false, true> : attn_prefix8_kernel<false, false>);
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, tq, p);
  if (e == cudaSuccess && plan.nsplit > 1) {
    cfg = pdl_config(dim3(static_cast<unsigned>((rows + kCombineWarps - 1) / kCombineWarps)), dim3(kCombineWarps * 32), 0,
                     stream, attr);
    e = cudaLaunchKernelEx(&cfg, attn_prefix8_combine_kernel, static_cast<const float*>(p.part_o),
                           static_cast<const float2*>(p.part_ml), plan.nsplit, rows, p.out, p.lse);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
