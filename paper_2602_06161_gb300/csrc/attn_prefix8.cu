// attn_prefix8.cu - two-view window attention over an 8-bit key/value memory.
//
// Query row r of head hq sits at memory position q0 + r and sees the keys lo <= j < hi of its row:
//   s_j = q . k_j / sqrt(d),  k_j = code * 2^(x - 127);  capped: s_j = c tanh(s_j / c)
//   o = sum_j softmax(s)_j v_j,  lse = ln sum_j e^{s_j}
// A seed row's own column, where it is among the row's keys, is the masked-input pair (k_i, v_i) instead
// (the leave-one-out view). A row that sees no key gives o = 0, lse = -inf; one that sees a key whose
// K or V row is NaN gives NaN.
//
// The G = Hq / Hkv query heads of a KV head are packed: row p = g Lq + r of KV head (b, hkv) is query row r of head
// hkv G + g, and the packed rows are one run of the [B Hq Lq, D] view. A CTA takes a group of them against the KV tiles (128
// keys) of one of nsplit parts of what its rows see; with nsplit > 1 the parts' CTAs are a cluster that adds up their (m, l, O)
// in fp32 itself (rows and tile, up to 8 parts), or leave them in the workspace for a second kernel (the rows kernels' parts
// of a batch with key ranges shared out to the sequences by their lengths, see share_of). Five ways, chosen by
// plan_of from the sizes:
//   rows (16 or 32 a group)  codes as 8-bit matrix operands, products turned over; bound by reading the memory
//   tile (128 rows)          codes decoded to bf16 by the CTA; bound by decoding
//   pairs (2 x 128 rows)     codes decoded once, by a pass of its own; bound by the tensor cores and the softmax
//   read back                the kernels of cover_attn_fwd_prefix over the decoded memory, without key ranges and caps
//
// The tile kernel. Codes arrive by bulk copies (128 rows are 16 KB in one piece); one warpgroup decodes K and one V to bf16
// (exact: a row's scale is a power of two) into the swizzled layout that the tensor cores read, and S = Q K^T, O += P V run as
// tcgen05.mma with S, P and O in tensor memory. Two softmax warpgroups keep one stream each: the even and the odd KV
// tiles, with sums and an accumulator of their own that are merged at the end, so that the chain load - decode - S - softmax -
// P V of one KV tile overlaps the next one's. A KV tile takes 1.34 us; the most of it is decoding: two instructions a
// code, and the 224 KB a tile that it, the look for NaN codes and the products move through shared memory take 0.9 us at 128 bytes a
// clock. Codes are looked through before their bf16 tile is free, where the decoding threads would wait (8 x 32 heads, 64 x
// 2048: 60 us; with the look inside the decoding 64, and 62 without any).
// Roles (640 threads): warps 0-3, 4-7 softmax of stream 0, 1 (thread = row); 8-11 decode K, 12-15 V; 16 issues the
// products; 17 and 18 the copies of K and V.
// Shared memory: Q (32 KB) | two tiles of K and of V codes (16 KB each) | K, V in bf16 (2 x 32 KB each).
// Tensor memory: S0 | S1 (P overwrites their first 64 columns) | O0 | O1, 128 columns each.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>
#include <cmath>

#include "cluster.cuh"
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
constexpr int kCodeBytes = kBN * kD;       // 16 KB of codes
constexpr int kHalf = kBN / 2;
constexpr int kThreads = 640;
constexpr int kDecodeWarp = 8, kMmaWarp = 16, kLoadWarp = 17;
constexpr int kLaunchRegs = 96;            // registers per thread at launch (65536 / 640, rounded down to 8)
// registers of the softmax, decode and issuing threads: a Q tile's softmax threads hold 128 scores each
constexpr int kSoftmaxRegs = 160, kDecodeRegs = 56, kIssueRegs = 40;
static_assert(2 * 128 * kSoftmaxRegs + 2 * 128 * kDecodeRegs + 128 * kIssueRegs <= kThreads * kLaunchRegs, "register split");
// setmaxnreg.inc takes no count below the thread's own, .dec none above it
static_assert(kSoftmaxRegs >= kLaunchRegs && kDecodeRegs <= kLaunchRegs && kIssueRegs <= kLaunchRegs, "register split");
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kMaxParts = 64;              // of the keys
constexpr int kMaxShared = 32;             // sequences that share the parts out by their lengths
constexpr int kMaxJoined = 8;              // parts whose CTAs are a cluster (its portable size)
constexpr int kSms = 152;                  // of this GPU; the split of the keys is chosen for it

// Barriers and tables of a CTA.
struct Ctl {
  uint64_t q_full;
  uint64_t c_full[2][2], c_empty[2][2]; // rings of K and V codes
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2], p_full[2];        // per stream
  uint64_t o_full, drain;
  uint32_t tmem_base;
  int abort;
  int lo, hi;                           // keys that some row of the CTA sees
  int wide;                             // a V row's byte is outside those that a fixed reference serves
  uint4 nan_keys[4];                    // per KV tile in turn: keys whose V row is NaN
};

struct Smem {
  uint8_t q[kTileBytes];
  uint8_t ring[4 * kCodeBytes];         // two tiles of K codes, two of V codes
  uint8_t k[2][kTileBytes];
  uint8_t v[2][kTileBytes];
  Ctl ctl;
  int slot[kBM];                        // seed slot of a row's position, or kNoSlot
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
  float* part_o;     // [nsplit][rows][128]; shared out by length: [slots + B][rows / B][128]
  float2* part_ml;   // as part_o's rows
  int2* shares;      // [B] shared out by length: a sequence's first slot and its slots; or null
  int* status;
  long long rows;    // B * Hq * Lq
  int B, n_seeds, Hq, Hkv, G, Lq, Lk, q0, n_groups, nsplit;
  int slots;         // parts of a KV head that the sequences share
  int joined;        // the parts' CTAs are a cluster and add their results up themselves
  float scale_log2;  // log2(e) / sqrt(d)
  float cap_log2;    // cap * log2(e)
  float cap_in;      // 2 log2(e) / (cap sqrt(d))
  float cap_x;       // 1 / (cap sqrt(d))
  float cap_poly[4]; // coefficients of the capped score's polynomial, in powers of 1 / (cap sqrt(d))
  float cap_ref;     // reference of all rows under a small cap, or -inf (see fixed_reference)
  uint32_t v_lo, v_hi;   // bytes of the V rows that it serves, in all four bytes
};

// The keys lo .. hi - 1 that row i of [B Lq] sees, held to 0 .. Lk: the bounds given may be any, and the tile and pairs kernels count
// columns of a KV tile from them. (The rows kernels compare positions with them, which no bound upsets; held at both
// ends there, a batch's tokens took 0.7 % longer.)
__device__ __forceinline__ int2 keys_of(const Params& p, size_t i) {
  const int lo = p.key_lo != nullptr ? __ldg(p.key_lo + i) : 0, hi = p.key_hi != nullptr ? __ldg(p.key_hi + i) : p.Lk;
  return make_int2(min(max(lo, 0), p.Lk), min(max(hi, 0), p.Lk));
}

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

// Bytes of x by the selector's nibbles; a nibble with its top bit set gives eight copies of that byte's sign.
template <uint32_t kSel>
__device__ __forceinline__ uint32_t prmt(uint32_t x) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(0), "n"(kSel));
  return d;
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

// Decodes a row of codes, eight 16-byte pieces, into its row of a bf16 tile (two 64-column boxes, 16-byte chunks swizzled by row & 7). An e4m3 code's bits s eeee mmm, moved to s 0000eeee mmm0000, are
// the bf16 number code * 2^-120 (subnormal codes included), and one multiplication by m1 = 2^(120 + x - 127) gives the
// value; where that is above bf16's range, m1 = 2^120 and kTwo says to multiply by m2 = 2^(x - 127) too. Both are
// exact. A row's pieces are taken in the order u0 ^ 0, u0 ^ 1, ... with u0 the row's low bits, so that the reads and writes
// of eight lanes meet every bank. src: address of piece u0; d0, d1: of its first chunk, in
// its box and in the other one.
template <bool kTwo>
__device__ __forceinline__ void decode_row(uint32_t src, uint32_t d0, uint32_t d1, uint32_t m1, uint32_t m2) {
#pragma unroll
  for (int i0 = 0; i0 < 8; i0 += 4) {
    uint4 c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = lds128(src ^ (16u * (i0 + i)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
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
      const uint32_t x = i0 + i;   // piece u0 ^ x
      const uint32_t d = (x & 4 ? d1 : d0) ^ ((x & 3) << 5);
      sts128(d, o[0], o[1], o[2], o[3]);
      sts128(d ^ 16u, o[4], o[5], o[6], o[7]);
    }
  }
}

// Whether a row of codes holds a NaN; src as in decode_row.
__device__ __forceinline__ bool nan_code(uint32_t src) {
  uint32_t hit = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 c = lds128(src ^ (16u * i));
    hit |= ((c.x & 0x7f7f7f7fu) + 0x01010101u) | ((c.y & 0x7f7f7f7fu) + 0x01010101u) | ((c.z & 0x7f7f7f7fu) + 0x01010101u) |
           ((c.w & 0x7f7f7f7fu) + 0x01010101u);
  }
  return (hit & 0x80808080u) != 0;
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
  if (__any_sync(0xffffffffu, two)) decode_row<true>(src, d0, d1, m1, m2);
  else decode_row<false>(src, d0, d1, m1, m2);
}

// The exponent bytes of row `row` of four KV tiles from tile j on (zero from row `left` of the part on).
struct FourBytes {
  uint32_t v[4];
  __device__ __forceinline__ void load(const uint8_t* exps, int j, int row, int left) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = (j + i) * kBN + row;
      v[i] = at < left ? __ldg(exps + at) : 0u;
    }
  }
  // (the asm keeps the compiler from packing them, and so waiting for the loads, where they are issued)
  __device__ __forceinline__ uint32_t packed() {
    asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]));
    return v[0] | (v[1] << 8) | (v[2] << 16) | (v[3] << 24);
  }
};

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

// Barriers and tensor memory, by one warp.
// fills: arrivals that fill a K or V tile (128 decoding threads, or the thread that issues its copies); rows: threads of a
// stream's softmax.
__device__ __forceinline__ void set_up(Ctl& ctl, const CUtensorMap* tm_q, uint32_t fills, uint32_t rows) {
  if ((threadIdx.x & 31) == 0) {
    mbar_init(&ctl.q_full, 1);
    for (int i = 0; i < 2; ++i) {
      for (int w = 0; w < 2; ++w) {
        mbar_init(&ctl.c_full[w][i], 1);
        mbar_init(&ctl.c_empty[w][i], 128);
      }
      mbar_init(&ctl.k_full[i], fills);
      mbar_init(&ctl.k_empty[i], 1);
      mbar_init(&ctl.v_full[i], fills);
      mbar_init(&ctl.v_empty[i], 1);
      mbar_init(&ctl.s_full[i], 1);
      mbar_init(&ctl.p_full[i], rows);
    }
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.drain, 1);
    ctl.abort = 0;
    ctl.lo = 0x7fffffff;
    ctl.hi = 0;
    ctl.wide = 0;
    fence_mbar_init();
    tma_prefetch_desc(tm_q);
  }
  __syncwarp();
  tmem_alloc(&ctl.tmem_base, 512);
  tmem_relinquish();
}

// Copies the codes of K (which = 0) or V (1) of KV tiles j0 .. j0 + nt - 1 through their ring of two tiles; one thread. With
// which = 0 its Q tiles are on their way to ctl.q_full already.
__device__ __forceinline__ void copy_codes(Ctl& ctl, const Params& p, int which, uint8_t* ring, size_t mem0, int j0, int nt) {
  const uint8_t* src = (which ? p.v8 : p.k8) + (mem0 + static_cast<size_t>(j0) * kBN) * kD;
  const uint32_t dst = smem_u32(ring) + which * 2 * kCodeBytes;
  int j = 0;
  bool ok = true;
  for (; j < nt; ++j) {
    const int st = j & 1;
    if (j >= 2) ok = mbar_wait(&ctl.c_empty[which][st], ((j >> 1) - 1) & 1, &ctl.abort);
    if (!ok) break;
    const uint32_t bytes = static_cast<uint32_t>(min(kBN, p.Lk - (j0 + j) * kBN)) * kD;
    mbar_arrive_expect_tx(&ctl.c_full[which][st], bytes);
    bulk_load(dst + st * kCodeBytes, src + static_cast<size_t>(j) * kCodeBytes, bytes, &ctl.c_full[which][st]);
  }
  if (!ok) {
    if (!ctl.abort) report_status(p.status, kStatusTimeout, 70);
    ctl.abort = 1;
  }
  // every copy lands before the CTA's shared memory is released, whatever the other roles did
  if (which == 0) mbar_wait(&ctl.q_full, 0, nullptr);
  for (int f = max(0, j - 2); f < j; ++f) mbar_wait(&ctl.c_full[which][f & 1], (f >> 1) & 1, nullptr);
}

// Decodes K (which = 0) or V (1) of KV tiles j0 .. j0 + nt - 1 into two bf16 tiles in turn; 128 threads, one a key.
__device__ __forceinline__ void decode_tiles(Ctl& ctl, const Params& p, int which, uint8_t* ring, uint8_t* k_tiles,
                                             uint8_t* v_tiles, size_t mem0, int j0, int nt) {
  const int row = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t u0 = static_cast<uint32_t>(row & 7);
  const uint32_t codes = smem_u32(ring) + which * 2 * kCodeBytes + row * kD + u0 * 16;
  const uint32_t tile = smem_u32(which ? v_tiles : k_tiles) + row * 128 + (((u0 & 3) << 5) ^ (u0 << 4));
  const uint32_t box = (u0 >> 2) * kBoxBytes;
  const int first = j0 * kBN;                    // this part's first key
  const int left = min(p.Lk - first, nt * kBN);  // keys of this part
  // exponent bytes are fetched four tiles at a time, four to eight ahead of their use
  const uint8_t* exps = (which ? p.v_exp : p.k_exp) + mem0 + first;
  FourBytes x_next;
  x_next.load(exps, 0, row, left);
  uint32_t xs = 0;
  bool ok = true;
  for (int j = 0; j < nt; ++j) {
    const int st = j & 1;
    if ((j & 3) == 0) {
      xs = x_next.packed();
      x_next.load(exps, j + 4, row, left);
    }
    const bool zero = j * kBN + row >= left;
    int x = (xs >> (8 * (j & 3))) & 255;
    // codes are looked through while the bf16 tile is still read
    ok = warp_wait(&ctl.c_full[which][st], (j >> 1) & 1, &ctl.abort);
    if (!ok) break;
    if (!zero && nan_code(codes + st * kCodeBytes)) x = kExpNan;
    const uint32_t nans = __ballot_sync(0xffffffffu, x > kExpMax);
    if (j >= 2) ok = warp_wait(which ? &ctl.v_empty[st] : &ctl.k_empty[st], ((j >> 1) - 1) & 1, &ctl.abort);
    if (!ok) break;
    // V: the softmax of tile j - 2, which read what stood here, is behind its products
    if (which && lane == 0) reinterpret_cast<uint32_t*>(&ctl.nan_keys[j & 3])[row >> 5] = nans;
    // a weight of zero times NaN is NaN: V rows of NaN are decoded as zeros, and the sums of the
    // rows that see their keys are made NaN instead
    const uint32_t to = tile + st * kTileBytes;
    decode(codes + st * kCodeBytes, to + box, to + (kBoxBytes - box), x, zero || (which && x > kExpMax));
    mbar_arrive(&ctl.c_empty[which][st]);
    fence_proxy_async_smem();
    mbar_arrive(which ? &ctl.v_full[st] : &ctl.k_full[st]);
  }
  if (!ok && lane == 0) {
    if (!ctl.abort) report_status(p.status, kStatusTimeout, 72);
    ctl.abort = 1;
  }
}

// This part's KV tiles among those that the CTA's rows see.
struct Part {
  int j0, nt;
};
__device__ __forceinline__ Part part_of(int lo, int hi, int ks, int nsplit) {
  const int t0 = hi > 0 ? lo / kBN : 0, t1 = hi > 0 ? (hi + kBN - 1) / kBN : 0;
  const int each = (t1 - t0) / nsplit, more = (t1 - t0) % nsplit;
  return Part{t0 + ks * each + min(ks, more), each + (ks < more ? 1 : 0)};
}

// Parts shared out to a batch's sequences by their lengths (rows kernels, with key ranges): of `slots` parts for a KV head every
// sequence gets as many as its KV tiles need for parts of at most t, and t is the least for which they are enough.
// Empty sequences have a part each, behind those. Returns the first part and the parts of sequence lane (all lanes
// of a warp; B <= 32, B <= slots).
__device__ __forceinline__ int2 share_of(const int* seq_lo, const int* seq_hi, int B, int slots) {
  const int lane = threadIdx.x & 31;
  int tiles = 0;
  if (lane < B && seq_hi[lane] > 0) tiles = (seq_hi[lane] + kBN - 1) / kBN - seq_lo[lane] / kBN;
  int hi = __reduce_max_sync(0xffffffffu, tiles), lo = max(1, (hi + kMaxParts - 1) / kMaxParts);   // t is among lo .. hi
  hi = max(hi, lo);
  while (lo < hi) {
    const int t = (lo + hi) / 2;
    if (__reduce_add_sync(0xffffffffu, (tiles + t - 1) / t) <= slots) hi = t;
    else lo = t + 1;
  }
  const int n = (tiles + hi - 1) / hi;
  int first = n;   // an inclusive sum over the sequences
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, first, d);
    if (lane >= d) first += x;
  }
  const int all = __shfl_sync(0xffffffffu, first, 31);
  const uint32_t empty = __ballot_sync(0xffffffffu, lane < B && n == 0);
  if (n > 0) return make_int2(first - n, n);
  return make_int2(all + __popc(empty & ((1u << lane) - 1u)), lane < B ? 1 : 0);
}

// What a row does not see of a KV tile: columns outside [lo, hi), its own one if it is a seed row (own, or -1); whether
// anything of it holds for some row of the warp.
struct Unseen {
  int lo, hi, own;
  bool any;
};

// Caps (to log2 units) and masks the scores of 32 columns from column c0 of the tile on. The loops over a row's chunks are
// not unrolled: with 128 columns at once 8 % of the instruction fetches missed the SM's cache, the GPC's was at 52 % of
// its rate, and a KV tile took 4950 cycles on 128 SMs where it took 2780 on 64.
template <bool kCap>
__device__ __forceinline__ void finish_scores(float (&s)[32], const Params& p, const Unseen& u, int c0) {
  if (kCap) {
#pragma unroll
    for (int c = 0; c < 32; ++c) s[c] = capped(s[c], p.cap_in, p.cap_log2);
  }
  if (u.any) {
    const int lo = u.lo - c0, hi = u.hi - c0, own = u.own - c0;
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (c < lo || c >= hi || c == own) s[c] = -INFINITY;
  }
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

// The largest of 32 columns' scores, neither scaled nor capped yet.
__device__ __forceinline__ float chunk_max(uint32_t addr, const Params& p, const Unseen& u, int c0) {
  uint32_t raw[32];
  tmem_ld32(addr, raw);
  tmem_ld_wait(raw);
  float(&s)[32] = reinterpret_cast<float(&)[32]>(raw);
  finish_scores<false>(s, p, u, c0);
  return max32(s);
}

// A row's reference in log2 units from its largest product (the cap is monotonous).
template <bool kCap>
__device__ __forceinline__ float reference_of(float top, const Params& p) {
  return !kCap ? top * p.scale_log2 : top == -INFINITY ? top : capped(top, p.cap_in, p.cap_log2);
}

// P = 2^(score - m) of 32 columns to tensor memory, in bf16: V's operands are, so P's have to be. A weight is off by at most 2^-8 of
// itself, as the output is of itself; TF32 operands would be exacter at half the rate. Returns the sum of the unrounded weights. fixed: capped scores whose reference is
// fixed; those of a chunk that are all small and all seen take the polynomial.
template <bool kCap>
__device__ __forceinline__ float chunk_exp(uint32_t addr, uint32_t p_addr, const Params& p, const Unseen& u, int c0, float m,
                                           bool fixed, bool valid) {
  uint32_t raw[32];
  tmem_ld32(addr, raw);
  tmem_ld_wait(raw);
  float(&s)[32] = reinterpret_cast<float(&)[32]>(raw);
  bool small = false;
  if (kCap) {
    if (fixed && !u.any) {
      float hi[2] = {};
#pragma unroll
      for (int c = 0; c < 32; c += 4) {
        hi[0] = fmax3(hi[0], fabsf(s[c]), fabsf(s[c + 1]));
        hi[1] = fmax3(hi[1], fabsf(s[c + 2]), fabsf(s[c + 3]));
      }
      small = __all_sync(0xffffffffu, fmaxf(hi[0], hi[1]) * p.cap_x <= kTanhRange || !valid);
    }
  }
  const uint64_t negm2 = f2_pack(-m, -m);
  uint64_t acc2[2] = {0, 0};
  uint32_t packed[16];
  if (kCap && small) {
    // C x P(x^2) with x = s cap_x, the powers of cap_x in the coefficients
    const uint64_t t0 = f2_pack(p.cap_poly[0], p.cap_poly[0]), t1 = f2_pack(p.cap_poly[1], p.cap_poly[1]),
                   t2 = f2_pack(p.cap_poly[2], p.cap_poly[2]), t3 = f2_pack(p.cap_poly[3], p.cap_poly[3]);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      const uint64_t x = f2_pack(s[2 * c], s[2 * c + 1]);
      const uint64_t z = f2_mul(x, x);
      float x0, x1;
      f2_unpack(f2_fma(x, f2_fma(z, f2_fma(z, f2_fma(z, t3, t2), t1), t0), negm2), x0, x1);
      const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
      packed[c] = pack_bf16x2(e0, e1);
      acc2[c & 1] = f2_add(acc2[c & 1], f2_pack(e0, e1));
    }
  } else {
    finish_scores<kCap>(s, p, u, c0);
    const float scale = kCap ? 1.0f : p.scale_log2;
    const uint64_t scale2 = f2_pack(scale, scale);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      float x0, x1;
      f2_unpack(f2_fma(f2_pack(s[2 * c], s[2 * c + 1]), scale2, negm2), x0, x1);
      const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
      packed[c] = pack_bf16x2(e0, e1);
      acc2[c & 1] = f2_add(acc2[c & 1], f2_pack(e0, e1));
    }
  }
  tmem_st16(p_addr, packed);
  float r[4];
  f2_unpack(acc2[0], r[0], r[1]);
  f2_unpack(acc2[1], r[2], r[3]);
  return (r[0] + r[1]) + (r[2] + r[3]);
}

// Whether V rows from .. to - 1 hold an exponent byte outside p.v_lo .. p.v_hi (bytes above 246, rows of NaN, are not meant: their values are
// taken as zeros); the part of it that thread tid of kAll looks at. exps: of row 0.
template <int kAll>
__device__ __forceinline__ bool bytes_outside(const Params& p, const uint8_t* exps, int from, int to, int tid) {
  constexpr uint32_t kNumbers = 0x01010101u * kExpMax;
  const uint8_t* bytes = exps + from;
  const int n = max(to - from, 0);
  const auto one = [&](int i) {
    const uint32_t x = __ldg(bytes + i);
    return x < (p.v_lo & 255u) || (x > (p.v_hi & 255u) && x <= kExpMax);
  };
  const auto four = [&](uint32_t x) { return __vcmpltu4(x, p.v_lo) | (__vcmpgtu4(x, p.v_hi) & __vcmpleu4(x, kNumbers)); };
  const int head = min(n, static_cast<int>(-reinterpret_cast<uintptr_t>(bytes) & 15)), wide = (n - head) / 16;
  uint32_t out = tid < head && one(tid) ? 1 : 0;
  for (int i = tid; i < wide; i += kAll) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(bytes + head) + i);
    out |= four(w.x) | four(w.y) | four(w.z) | four(w.w);
  }
  const int last = head + 16 * wide + tid;
  return out != 0 || (last < n && one(last));
}

// A seed row's own score in log2 units: q row `row` of [B Hq Lq], masked-input key row `self`.
template <bool kCap>
__device__ __forceinline__ float self_score(const Params& p, long long row, size_t self) {
  const uint4* qr = reinterpret_cast<const uint4*>(p.q + row * kD);
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
  return kCap ? capped(d0 + d1, p.cap_in, p.cap_log2) : (d0 + d1) * p.scale_log2;
}

// A row's sum l under a fixed reference m, which may be far from the row's scores: the sum goes to [1, 2), the reference with it
// (to -inf for a sum of zero: a row or a part without keys), and the accumulator's factor, 2 to a whole number, is returned. So a row's
// reference is that of its largest weights within the sum's bits when it meets those of other parts and of the masked-input
// pair, whose values may be of any size.
__device__ __forceinline__ float follow_sum(float& m, float& l) {
  if (l == 0.0f) m = -INFINITY;
  const int e = static_cast<int>(__float_as_uint(l) >> 23);   // (l > 0 is a normal number)
  if (e == 0 || e == 255) return 1.0f;
  m += static_cast<float>(e - 127);
  const float f = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
  l *= f;
  return f;
}

// o += w v for 32 columns of a masked-input value.
__device__ __forceinline__ void add_self(float (&o)[32], float w, const __nv_bfloat16* v) {
  const uint4* vr = reinterpret_cast<const uint4*>(v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint4 a = __ldg(vr + e);
    const uint32_t x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      o[8 * e + 2 * f] = fmaf(w, __uint_as_float(x[f] << 16), o[8 * e + 2 * f]);
      o[8 * e + 2 * f + 1] = fmaf(w, __uint_as_float(x[f] & 0xffff0000u), o[8 * e + 2 * f + 1]);
    }
  }
}

// 32 columns of a row: a part's accumulator, or the result (a NaN sum makes the whole row NaN).
__device__ __forceinline__ void store_chunk(const Params& p, const float (&o)[32], float inv, bool split, int ks, long long orow,
                                            int col) {
  if (split) {
    float4* dst = reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(ks) * p.rows + orow) * kD + col);
#pragma unroll
    for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
  } else {
    uint4* dst = reinterpret_cast<uint4*>(p.out + orow * kD + col);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      dst[e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                          pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
  }
}

// Parts that a cluster's CTAs add up themselves: each stages its rows' accumulators [row][128] fp32 and (m, l) in its own
// shared memory, and CTA ks finishes the rows ks, ks + nsplit, .., a warp a row, reading all CTAs'. Rows' 16-byte
// pieces are swizzled, for the threads that write a row each.
__device__ __forceinline__ uint32_t staged_at(int row, int c4) { return row * (kD * 4) + ((c4 ^ (row & 31)) << 4); }

__device__ __forceinline__ float4 lds_cluster128(uint32_t addr) {
  float4 r;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "r"(addr) : "memory");
  return r;
}
__device__ __forceinline__ float2 lds_cluster64(uint32_t addr) {
  float2 r;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(addr) : "memory");
  return r;
}

// kPad: nsplit rounded up to 4 or 8. A warp works on kBatch rows at once.
template <int kPad, int kBatch>
__device__ __forceinline__ void join_rows(const Params& p, uint32_t o, uint32_t ml, int n_rows, long long orow0, int ks) {
  static_assert(kPad * kBatch <= 32, "a lane for every part of the rows at work");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int first = ks + p.nsplit * warp; first < n_rows; first += 8 * p.nsplit * kBatch) {
    // lane: part lane % kPad of the batch's row lane / kPad (row numbers past the last one are held to it)
    const auto row = [&](int i) { return min(first + 8 * p.nsplit * i, n_rows - 1); };
    const int j = lane % kPad;
    const float2 part = lds_cluster64(cluster_map(ml + 8 * row(min(lane / kPad, kBatch - 1)), min(j, p.nsplit - 1)));
    float4 x[kBatch][kPad];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
#pragma unroll
      for (int k = 0; k < kPad; ++k) {
        x[i][k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k < p.nsplit) x[i][k] = lds_cluster128(cluster_map(o + staged_at(row(i), lane), k));
      }
    const float my_m = j < p.nsplit ? part.x : -INFINITY;
    float m = my_m;
#pragma unroll
    for (int d = kPad / 2; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float half = my_m == -INFINITY ? 0.0f : ex2_approx(0.5f * (my_m - m)), w = half * half;
    float l = j < p.nsplit ? half * part.y * half : 0.0f;
#pragma unroll
    for (int d = kPad / 2; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int n = first + 8 * p.nsplit * i;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kPad; ++k) {
        const float wk = __shfl_sync(0xffffffffu, w, i * kPad + k);   // (parts that saw no key hold zeros)
        acc.x = fmaf(wk, x[i][k].x, acc.x);
        acc.y = fmaf(wk, x[i][k].y, acc.y);
        acc.z = fmaf(wk, x[i][k].z, acc.z);
        acc.w = fmaf(wk, x[i][k].w, acc.w);
      }
      const float f = __shfl_sync(0xffffffffu, inv, i * kPad);
      if (n < n_rows)
        reinterpret_cast<uint2*>(p.out + (orow0 + n) * kD)[lane] =
            make_uint2(pack_bf16x2(acc.x * f, acc.y * f), pack_bf16x2(acc.z * f, acc.w * f));
    }
    const int n = first + 8 * p.nsplit * (lane / kPad);
    if (p.lse != nullptr && j == 0 && lane / kPad < kBatch && n < n_rows) p.lse[orow0 + n] = (m + lg2_approx(l)) * 0.6931471805599453f;
  }
}

// kMany: Q tiles of 128 rows, whose warps have 2 rows and more to finish: four of four parts at once, or two (1 x 32 heads,
// 256 x 1024, two parts: 17.7 us with one row after the other, 16.0 us so). With 16 or 32 rows a warp has one
// or two; there the longer code costs more than it saves (rows of 32: 10.4 against 11.3 us).
template <bool kMany>
__device__ __forceinline__ void join_parts(const Params& p, uint32_t o, uint32_t ml, int n_rows, long long orow0, int ks) {
  __syncwarp();
  cluster_sync();   // every CTA's rows are staged
  if (kMany && p.nsplit <= 4) join_rows<4, 4>(p, o, ml, n_rows, orow0, ks);
  else join_rows<8, kMany ? 2 : 1>(p, o, ml, n_rows, orow0, ks);
  __syncwarp();
  cluster_sync();   // no CTA leaves while its rows are read
}
// The other roles' warps take part in the cluster's barriers.
__device__ __forceinline__ void join_pass() {
  __syncwarp();
  cluster_sync();
  cluster_sync();
}

// All 512 softmax threads of the pairs kernel.
__device__ __forceinline__ void pairs_sync() { asm volatile("bar.sync 1, 512;" ::: "memory"); }

// Barrier of one Q tile's 256 softmax threads of the pairs kernel, and with the vote whether any of them says so.
__device__ __forceinline__ void tile_sync(int tile) { asm volatile("bar.sync %0, 256;" ::"r"(2 + tile) : "memory"); }
__device__ __forceinline__ bool tile_any(int tile, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, 256, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(x ? 1u : 0u), "r"(2 + tile)
      : "memory");
  return r != 0;
}

template <bool kCap>
__global__ void __launch_bounds__(kThreads, 1)
    attn_prefix8_tile_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Ctl& ctl = sm.ctl;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // CTA (ks, group, hkv, b)
  const int ks = static_cast<int>(blockIdx.x) % p.nsplit;
  int rest = static_cast<int>(blockIdx.x) / p.nsplit;
  const int group = rest % p.n_groups;
  rest /= p.n_groups;
  const int hkv = rest % p.Hkv;
  const int b = rest / p.Hkv;
  const int n_packed = p.G * p.Lq;
  const int p0 = group * kBM;                                                         // the CTA's first packed row
  const long long rowbase = (static_cast<long long>(b) * p.Hq + hkv * p.G) * p.Lq;    // packed row 0 in [B Hq Lq, D]
  const size_t mem0 = (static_cast<size_t>(b) * p.Hkv + hkv) * p.Lk;                  // the KV head's first memory row

  if (warp == kMmaWarp) set_up(ctl, &tm_q, 128, 128);
  if (p.n_seeds > 0 && tid < kBM) sm.slot[tid] = kNoSlot;
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = ctl.tmem_base;
  griddep_wait();
  griddep_launch_dependents();

  // ---------------- the rows' keys ----------------
  // softmax thread: its row, the keys [row_lo, row_hi) that it sees
  const int stream = warp >> 2;                       // of a softmax warp
  const int R = tid & (kBM - 1);
  const int P = p0 + R;
  const bool valid = warp < kDecodeWarp && P < n_packed;
  const int r = valid ? P % p.Lq : 0;
  int row_lo = 0, row_hi = p.Lk;
  if (valid) {
    const int2 keys = keys_of(p, static_cast<size_t>(b) * p.Lq + r);
    row_lo = keys.x, row_hi = keys.y;
  }
  int lo_key = 0, hi_key = p.Lk;                      // keys that some row sees
  if (p.key_lo != nullptr || p.key_hi != nullptr) {
    if (warp < kDecodeWarp) {
      const bool some = valid && row_lo < row_hi;
      const int lo = __reduce_min_sync(0xffffffffu, some ? row_lo : 0x7fffffff);
      const int hi = __reduce_max_sync(0xffffffffu, some ? row_hi : 0);
      if (lane == 0 && hi > 0) {
        atomicMin(&ctl.lo, lo);
        atomicMax(&ctl.hi, hi);
      }
    }
    __syncthreads();
    lo_key = ctl.lo, hi_key = ctl.hi;
  }
  const Part part = part_of(lo_key, hi_key, ks, p.nsplit);
  const int j0 = part.j0, nt = part.nt;

  if (warp >= kMmaWarp) {
    setmaxnreg_dec<kIssueRegs>();
    if ((warp == kLoadWarp || warp == kLoadWarp + 1) && lane == 0 && nt > 0) {
      if (warp == kLoadWarp) {
        mbar_arrive_expect_tx(&ctl.q_full, kTileBytes);
        for (int h = 0; h < 2; ++h)
          tma_load_4d(sm.q + h * kBoxBytes, &tm_q, &ctl.q_full, 64 * h, static_cast<int>(rowbase) + p0, 0, 0);
      }
      copy_codes(ctl, p, warp - kLoadWarp, sm.ring, mem0, j0, nt);
    } else if (warp == kMmaWarp && lane == 0 && nt > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_qk = idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t id_pv = idesc_bf16_f32(kBM, kD, false, true);
      constexpr uint64_t kTileDesc = kTileBytes >> 4;
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q), 16, 1024);
      const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
      const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), kBoxBytes, 1024);
      // S[s] = Q . K(stage)^T
      auto issue_s = [&](int s, int st) {
        uint64_t a = dq, kb = dk + st * kTileDesc;
        asm volatile("" : "+l"(a), "+l"(kb));   // descriptors are added up here, not kept in registers
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          const uint64_t off = static_cast<uint64_t>(((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4);
          umma_ss(tbase + s * kBN, a + off, kb + off, id_qk, kk > 0 ? 1u : 0u);
        }
        umma_commit(&ctl.s_full[s]);
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
        const bool ok = mbar_wait(bar, phase & 1, &ctl.abort);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      bool ok = wait(&ctl.q_full, 0);
      // stream j & 1 takes tile j, from stage j & 1
      for (int j = 0; j < 2 && j < nt && ok; ++j) {
        ok = wait(&ctl.k_full[j], 0);
        if (!ok) break;
        issue_s(j, j);
        umma_commit(&ctl.k_empty[j]);
      }
      for (int j = 0; j < nt && ok; ++j) {
        const int s = j & 1;
        ok = wait(&ctl.v_full[s], j >> 1) && wait(&ctl.p_full[s], j >> 1);
        if (!ok) break;
        issue_pv(s, s, j > 1);
        umma_commit(&ctl.v_empty[s]);
        if (j + 2 < nt) {
          ok = wait(&ctl.k_full[s], (j + 2) >> 1);
          if (!ok) break;
          issue_s(s, s);
          umma_commit(&ctl.k_empty[s]);
        }
      }
      if (ok) {
        umma_commit(&ctl.o_full);
      } else {
        if (!ctl.abort) report_status(p.status, kStatusTimeout, 71);
        ctl.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&ctl.drain);
      mbar_wait(&ctl.drain, 0, nullptr);
    }
    __syncwarp();
    if (p.joined) join_pass();
  } else if (warp >= kDecodeWarp) {
    setmaxnreg_dec<kDecodeRegs>();
    decode_tiles(ctl, p, (warp - kDecodeWarp) >> 2, sm.ring, sm.k[0], sm.v[0], mem0, j0, nt);
    if (p.joined) join_pass();
  } else {
    // ---------------- softmax ----------------
    setmaxnreg_inc<kSoftmaxRegs>();
    int slot = kNoSlot;
    if (p.n_seeds > 0) {
      // the CTA's rows stand at up to 128 positions: r itself, or r - r0 around Lq
      const int r0 = p.Lq <= kBM ? 0 : p0 % p.Lq;
      const int32_t* seeds = p.seed_idx + static_cast<size_t>(b) * p.n_seeds;
      for (int s = tid; s < p.n_seeds; s += 2 * kBM) {
        const int at = __ldg(seeds + s) - p.q0;
        if (at < 0 || at >= p.Lq) continue;
        const int i = at >= r0 ? at - r0 : at - r0 + p.Lq;
        if (i < kBM) atomicMin(&sm.slot[i], s);
      }
      softmax_sync();
      if (valid) slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq];
    }
    const int pos = p.q0 + r;
    const bool is_seed = slot != kNoSlot;
    const bool warp_seed = __any_sync(0xffffffffu, is_seed);
    const size_t self = (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds + (is_seed ? slot : 0);
    // the seed rows' own scores (log2 units), in the first part alone
    const float s_self = ks == 0 && is_seed && pos >= row_lo && pos < row_hi
                             ? self_score<kCap>(p, rowbase + P, self) : -INFINITY;
    const bool warp_live = __any_sync(0xffffffffu, valid);
    const uint32_t s_addr = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16) + stream * kBN;
    const uint32_t o_addr = s_addr + 2 * kBN;
    // a reference of all rows where the part's V rows, those that some row sees, allow it
    bool fixed = kCap && p.cap_ref != -INFINITY;
    if (fixed) {
      if (bytes_outside<2 * kBM>(p, p.v_exp + mem0, max(lo_key, j0 * kBN), min(hi_key, (j0 + nt) * kBN), tid)) ctl.wide = 1;
      softmax_sync();
      fixed = ctl.wide == 0;
    }
    float m_run = fixed ? p.cap_ref : -INFINITY, l_run = 0.0f;
    bool ok = true;
    // A row that sees a key whose V row is NaN has a NaN sum. V is decoded beside K, and that its tile is behind the softmax of the
    // keys is no matter: the rows are known when its products are (waiting for them before took 5 % of a call).
    const auto nan_values = [&](int t) {
      const uint32_t* nan = reinterpret_cast<const uint32_t*>(&ctl.nan_keys[t & 3]);
#pragma unroll 1
      for (int w = 0; w < 4; ++w) {
        for (uint32_t bits = nan[w]; bits != 0; bits &= bits - 1) {
          const int at = (j0 + t) * kBN + 32 * w + __ffs(bits) - 1;
          if (at >= row_lo && at < row_hi && !(is_seed && at == pos)) l_run = __uint_as_float(0x7fc00000u);
        }
      }
    };
    int i = 0;   // the stream's step
    for (int j = stream; j < nt; j += 2, ++i) {
      ok = warp_wait(&ctl.s_full[stream], i & 1, &ctl.abort);
      if (!ok) break;
      tc_fence_after_sync();
      if (i > 0) nan_values(j - 2);   // its products were issued before this S, and V's tile j + 2 waits for this one's
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
        mbar_arrive(&ctl.p_full[stream]);
        continue;
      }
      const bool own_column = warp_seed && __any_sync(0xffffffffu, is_seed && pos >= key0 && pos < key0 + kBN);
      const Unseen u{cl, ch, is_seed ? pos - key0 : -1, own_column || __any_sync(0xffffffffu, valid && (cl > 0 || ch < kBN))};
      float alpha = 1.0f;
      bool rescaled = false;
      if (!fixed) {
        float m_tile = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < kBN; c += 32) m_tile = fmaxf(m_tile, chunk_max(s_addr + c, p, u, c));
        m_tile = reference_of<kCap>(m_tile, p);
        if (m_tile > m_run + kRescaleThreshold) {
          alpha = (m_run == -INFINITY) ? 0.0f : ex2_approx(m_run - m_tile);
          m_run = m_tile;
          rescaled = true;
        }
      }
      const float m_use = (m_run == -INFINITY) ? 0.0f : m_run;
      l_run *= alpha;
#pragma unroll 1
      for (int c = 0; c < kBN; c += 32)
        l_run += chunk_exp<kCap>(s_addr + c, s_addr + c / 2, p, u, c, m_use, fixed, valid);
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
      mbar_arrive(&ctl.p_full[stream]);
    }
    if (ok && nt > 0) ok = warp_wait(&ctl.o_full, 0, &ctl.abort);
    if (ok && i > 0) nan_values(stream + 2 * (i - 1));
    if (!ok && lane == 0) {
      if (!ctl.abort) report_status(p.status, kStatusTimeout, 73);
      ctl.abort = 1;
    }

    // ---------------- the rows' results ----------------
    // of the thread's row: the sums of the streams that worked on it, and the accumulators' weights
    tc_fence_after_sync();
    const uint32_t o0 = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 2 * kBN;
    float2* ml = reinterpret_cast<float2*>(sm.q);   // every product is complete: Q is not read any more
    if (ok) ml[stream * kBM + R] = make_float2(m_run, l_run);
    softmax_sync();
    const float2 ml0 = ml[R], ml1 = ml[kBM + R];
    float m = fmaxf(ml0.x, ml1.x);
    const float m_use = m == -INFINITY ? 0.0f : m;
    float w[2] = {ml0.x == -INFINITY ? 0.0f : ex2_approx(ml0.x - m_use), ml1.x == -INFINITY ? 0.0f : ex2_approx(ml1.x - m_use)};
    float l = w[0] * ml0.y + w[1] * ml1.y;
    if (fixed) {
      const float f = follow_sum(m, l);
      w[0] *= f, w[1] *= f;
    }
    const int c0 = 2 * stream;   // the first of two 32-column chunks that this thread finishes
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
    const long long orow = rowbase + P;
    const bool split = p.nsplit > 1;
    const uint32_t staged = smem_u32(sm.k);   // nor are K's tiles
    // 1 / l, once a row; zero where no key was seen
    const float inv = split ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
    if (ok && warp_live) {
#pragma unroll 1
      for (int c = c0; c < c0 + 2; ++c) {
        float o[32];
        if (nt > 0) {
          uint32_t x[32];
          tmem_ld32(o0 + 32 * c, x);
          tmem_ld_wait(x);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = w[0] == 0.0f ? 0.0f : __uint_as_float(x[e]) * w[0];
          if (nt > 1) {
            tmem_ld32(o0 + kD + 32 * c, x);
            tmem_ld_wait(x);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(x[e]), w[1], o[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.0f;
        }
        if (p_self != 0.0f) add_self(o, p_self, p.v_seedmask + self * kD + 32 * c);
        if (valid && p.joined) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sts128(staged + staged_at(R, 8 * c + e), __float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]),
                   __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3]));
        } else if (valid) {
          store_chunk(p, o, inv, split, ks, orow, 32 * c);
        }
        __syncwarp();   // the next chunk is loaded by the whole warp
      }
      if (valid && c0 == 0) {
        if (p.joined) ml[2 * kBM + R] = make_float2(m, l);
        else if (split) p.part_ml[static_cast<size_t>(ks) * p.rows + orow] = make_float2(m, l);
        else if (p.lse != nullptr) p.lse[orow] = (m + lg2_approx(l)) * 0.6931471805599453f;
      }
    }
    tc_fence_before_sync();
    if (p.joined) join_parts<true>(p, staged, smem_u32(ml + 2 * kBM), min(kBM, n_packed - p0), rowbase + p0, ks);
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, 512);
  }
}

// ---------------------------------------------------------------------------
// Many rows
// ---------------------------------------------------------------------------
// A memory that many Q tiles read is decoded once, into the workspace (a row whose K or V is NaN has a NaN key and a zero
// value there), and a CTA takes two Q tiles, one a stream, that read each KV tile together. Two threads of different
// warpgroups share a row, 64 columns each, in two chunks of 32. 2048 rows over 8192 keys, 32 / 8 heads: 222 us, capped
// at 30 252 (8 us of them decode the memory); 1216 rows, which fill the GPU's 152 SMs once, 116 us, 1400 TFLOP/s: a KV tile takes
// 1.6 us, the products 1.1 of them; each Q tile's chain (S, maxima, exponentials, P V) is longer than the other's products. With a
// thread a row and its 128 columns unrolled it was 235 and 333 us: see finish_scores. One CTA an SM that walks over even shares of all
// tiles, units cut where a share ends, was tried: 1216 rows 130 us (a KV tile takes 0.1 us longer in such a loop), 2048 232 and 263.
// Roles (640 threads): warps 0-15 softmax (warpgroup 2 t + h: columns 64 h .. 64 h + 63 of Q tile t); 16 products; 17, 18
// copies of K, V.
// P of a half overwrites the first 32 columns of that half's scores, behind its loads.
constexpr int kPairSoftmaxWarps = 16, kPairMmaWarp = 16, kPairLoadWarp = 17;

struct PairSmem {
  uint8_t q[2][kTileBytes];
  uint8_t k[2][kTileBytes];
  uint8_t v[2][kTileBytes];
  Ctl ctl;
  float red[2][2][kBM];                 // per Q tile and half of the columns
  int slot[2 * kBM];                    // seed slot of a row's position, or kNoSlot
};

// Copies K (which = 0) or V (1) of KV tiles j0 .. j0 + nt - 1, decoded already, into the two bf16 tiles in turn; one thread.
__device__ __forceinline__ void copy_tiles(Ctl& ctl, const Params& p, int which, const CUtensorMap* tm, uint8_t* tiles, int hkv,
                                           int b, int j0, int nt) {
  uint64_t* const full = which ? ctl.v_full : ctl.k_full;
  uint64_t* const empty = which ? ctl.v_empty : ctl.k_empty;
  int j = 0;
  bool ok = true;
  for (; j < nt; ++j) {
    const int st = j & 1;
    if (j >= 2) ok = mbar_wait(&empty[st], ((j >> 1) - 1) & 1, &ctl.abort);
    if (!ok) break;
    mbar_arrive_expect_tx(&full[st], kTileBytes);
    for (int h = 0; h < 2; ++h)
      tma_load_4d(tiles + st * kTileBytes + h * kBoxBytes, tm, &full[st], 64 * h, (j0 + j) * kBN, hkv, b);
  }
  if (!ok) {
    if (!ctl.abort) report_status(p.status, kStatusTimeout, 76);
    ctl.abort = 1;
  }
  // every copy lands before the CTA's shared memory is released, whatever the other roles did
  if (which == 0) mbar_wait(&ctl.q_full, 0, nullptr);
  for (int f = max(0, j - 2); f < j; ++f) mbar_wait(&full[f & 1], (f >> 1) & 1, nullptr);
}

template <bool kCap>
__global__ void __launch_bounds__(kThreads, 1)
    attn_prefix8_pairs_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                              const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  PairSmem& sm = *reinterpret_cast<PairSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Ctl& ctl = sm.ctl;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // CTA (ks, group, hkv, b)
  const int ks = static_cast<int>(blockIdx.x) % p.nsplit;
  int rest = static_cast<int>(blockIdx.x) / p.nsplit;
  const int group = rest % p.n_groups;
  rest /= p.n_groups;
  const int hkv = rest % p.Hkv;
  const int b = rest / p.Hkv;
  const int n_packed = p.G * p.Lq;
  const int p0 = group * 2 * kBM;
  const long long rowbase = (static_cast<long long>(b) * p.Hq + hkv * p.G) * p.Lq;

  if (warp == kPairMmaWarp) set_up(ctl, &tm_q, 1, 256);
  if (p.n_seeds > 0 && tid < 2 * kBM) sm.slot[tid] = kNoSlot;
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = ctl.tmem_base;
  griddep_wait();
  griddep_launch_dependents();

  // ---------------- the rows' keys ----------------
  const int tile = warp >> 3, half = (warp >> 2) & 1;   // of a softmax warp
  const int R = tid & (kBM - 1);
  const int P = p0 + tile * kBM + R;
  const bool valid = warp < kPairSoftmaxWarps && P < n_packed;
  const int r = valid ? P % p.Lq : 0;
  int row_lo = 0, row_hi = p.Lk;
  if (valid) {
    const int2 keys = keys_of(p, static_cast<size_t>(b) * p.Lq + r);
    row_lo = keys.x, row_hi = keys.y;
  }
  int lo_key = 0, hi_key = p.Lk;                        // keys that some row sees
  if (p.key_lo != nullptr || p.key_hi != nullptr) {
    if (warp < kPairSoftmaxWarps) {
      const bool some = valid && row_lo < row_hi;
      const int lo = __reduce_min_sync(0xffffffffu, some ? row_lo : 0x7fffffff);
      const int hi = __reduce_max_sync(0xffffffffu, some ? row_hi : 0);
      if (lane == 0 && hi > 0) {
        atomicMin(&ctl.lo, lo);
        atomicMax(&ctl.hi, hi);
      }
    }
    __syncthreads();
    lo_key = ctl.lo, hi_key = ctl.hi;
  }
  const Part part = part_of(lo_key, hi_key, ks, p.nsplit);
  const int j0 = part.j0, nt = part.nt;
  const bool two_tiles = p0 + kBM < n_packed;           // the second Q tile has rows

  if (warp >= kPairMmaWarp) {
    if ((warp == kPairLoadWarp || warp == kPairLoadWarp + 1) && lane == 0 && nt > 0) {
      const int which = warp - kPairLoadWarp;
      if (which == 0) {
        mbar_arrive_expect_tx(&ctl.q_full, 2 * kTileBytes);
        for (int t = 0; t < 2; ++t)
          for (int h = 0; h < 2; ++h)
            tma_load_4d(sm.q[t] + h * kBoxBytes, &tm_q, &ctl.q_full, 64 * h, static_cast<int>(rowbase) + p0 + t * kBM, 0, 0);
      }
      copy_tiles(ctl, p, which, which ? &tm_v : &tm_k, which ? sm.v[0] : sm.k[0], hkv, b, j0, nt);
    } else if (warp == kPairMmaWarp && lane == 0 && nt > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_qk = idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t id_pv = idesc_bf16_f32(kBM, kD, false, true);
      constexpr uint64_t kTileDesc = kTileBytes >> 4;
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[0]), 16, 1024);
      const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
      const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), kBoxBytes, 1024);
      const uint32_t q_lo = static_cast<uint32_t>(dq), k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv);
      const uint32_t qk_hi = static_cast<uint32_t>(dq >> 32), v_hi = static_cast<uint32_t>(dv >> 32);
      // What this thread does between a barrier and its products is on every tile's way: descriptors are added up in their
      // lower words, and of several barriers the one that completes last is waited for last (1216 rows over 8192 keys 124 -> 116 us).
      // A thread for each Q tile took 170 us, P taken in two pieces as its chunks get ready 131, a thread that polls its barriers
      // 129, the two Q tiles' softmax in turns 122 to 126.
      const auto desc = [](uint32_t lo, uint32_t hi) { return (static_cast<uint64_t>(hi) << 32) | lo; };
      // S[s] = Q[s] . K(stage)^T
      auto issue_s = [&](int s, int st) {
        const uint32_t a = q_lo + s * static_cast<uint32_t>(kTileDesc), kb = k_lo + st * static_cast<uint32_t>(kTileDesc);
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          const uint32_t off = static_cast<uint32_t>(((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4);
          umma_ss(tbase + s * kBN, desc(a + off, qk_hi), desc(kb + off, qk_hi), id_qk, kk > 0 ? 1u : 0u);
        }
        umma_commit(&ctl.s_full[s]);
      };
      // O[s] (+)= P[s] . V(stage)
      auto issue_pv = [&](int s, int st, bool acc) {
        const uint32_t vb = v_lo + st * static_cast<uint32_t>(kTileDesc);
#pragma unroll
        for (int kk = 0; kk < kBN / 16; ++kk)
          umma_ts(tbase + 2 * kBN + s * kD, tbase + s * kBN + (kk >> 2) * kHalf + 8 * (kk & 3),
                  desc(vb + static_cast<uint32_t>((kk * 2048) >> 4), v_hi), id_pv, (acc || kk > 0) ? 1u : 0u);
      };
      auto wait = [&](uint64_t* bar, int phase) {
        const bool ok = mbar_wait(bar, phase & 1, &ctl.abort);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      bool ok = wait(&ctl.q_full, 0);
      if (ok && (ok = wait(&ctl.k_full[0], 0))) {
        issue_s(0, 0);
        if (two_tiles) issue_s(1, 0);
        umma_commit(&ctl.k_empty[0]);
      }
      for (int j = 0; j < nt && ok; ++j) {
        const int st = j & 1;
        const bool next = j + 1 < nt;
        ok = (!next || wait(&ctl.k_full[st ^ 1], (j + 1) >> 1)) && wait(&ctl.v_full[st], j >> 1) && wait(&ctl.p_full[0], j);
        if (!ok) break;
        issue_pv(0, st, j > 0);
        if (next) issue_s(0, st ^ 1);
        if (two_tiles) {
          ok = wait(&ctl.p_full[1], j);
          if (!ok) break;
          issue_pv(1, st, j > 0);
          if (next) issue_s(1, st ^ 1);
        }
        umma_commit(&ctl.v_empty[st]);
        if (next) umma_commit(&ctl.k_empty[st ^ 1]);
      }
      if (ok) {
        umma_commit(&ctl.o_full);
      } else {
        if (!ctl.abort) report_status(p.status, kStatusTimeout, 77);
        ctl.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&ctl.drain);
      mbar_wait(&ctl.drain, 0, nullptr);
    }
    __syncwarp();
  } else {
    // ---------------- softmax ----------------
    int slot = kNoSlot;
    if (p.n_seeds > 0) {
      // the CTA's rows stand at up to 256 positions: r itself, or r - r0 around Lq
      const int r0 = p.Lq <= 2 * kBM ? 0 : p0 % p.Lq;
      const int32_t* seeds = p.seed_idx + static_cast<size_t>(b) * p.n_seeds;
      for (int s = tid; s < p.n_seeds; s += 4 * kBM) {
        const int at = __ldg(seeds + s) - p.q0;
        if (at < 0 || at >= p.Lq) continue;
        const int i = at >= r0 ? at - r0 : at - r0 + p.Lq;
        if (i < 2 * kBM) atomicMin(&sm.slot[i], s);
      }
      pairs_sync();
      if (valid) slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq];
    }
    const int pos = p.q0 + r;
    const bool is_seed = slot != kNoSlot;
    const bool warp_seed = __any_sync(0xffffffffu, is_seed);
    const size_t self = (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds + (is_seed ? slot : 0);
    const float s_self = ks == 0 && is_seed && pos >= row_lo && pos < row_hi
                             ? self_score<kCap>(p, rowbase + P, self) : -INFINITY;
    const bool warp_live = __any_sync(0xffffffffu, valid);
    const uint32_t quad = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = quad + tile * kBN + half * kHalf;
    const uint32_t o_addr = quad + 2 * kBN + tile * kD + half * kHalf;
    // a reference of all rows where the part's V rows, those that some row sees, allow it
    bool fixed = kCap && p.cap_ref != -INFINITY;
    if (fixed) {
      const uint8_t* exps = p.v_exp + (static_cast<size_t>(b) * p.Hkv + hkv) * p.Lk;
      if (bytes_outside<4 * kBM>(p, exps, max(lo_key, j0 * kBN), min(hi_key, (j0 + nt) * kBN), tid)) ctl.wide = 1;
      pairs_sync();
      fixed = ctl.wide == 0;
    }
    float m_run = fixed ? p.cap_ref : -INFINITY, l_run = 0.0f;
    bool ok = true;
    const int jend = tile == 1 && !two_tiles ? 0 : nt;
    for (int j = 0; j < jend; ++j) {
      ok = warp_wait(&ctl.s_full[tile], j & 1, &ctl.abort);
      tc_fence_after_sync();   // zeros are stored over S too, where no row sees a key
      const int key0 = (j0 + j) * kBN + half * kHalf;
      const int cl = row_lo - key0, ch = row_hi - key0;   // columns cl <= c < ch of this half are seen
      // (a warp none of whose rows sees a key here stores zeros; a row without a query row may hold anything)
      const bool some = __any_sync(0xffffffffu, valid && max(cl, 0) < min(ch, kHalf));
      const bool own_column = warp_seed && __any_sync(0xffffffffu, is_seed && pos >= key0 && pos < key0 + kHalf);
      const Unseen u{cl, ch, is_seed ? pos - key0 : -1, own_column || __any_sync(0xffffffffu, valid && (cl > 0 || ch < kHalf))};
      float m_half = -INFINITY;
      if (ok && some && !fixed) {
#pragma unroll 1
        for (int c = 0; c < kHalf; c += 32) m_half = fmaxf(m_half, chunk_max(s_addr + c, p, u, c));
        m_half = reference_of<kCap>(m_half, p);
      }
      if (fixed && !ok) break;
      // The Q tile's 256 threads vote: a warp whose wait gave up takes part all the same, and both halves of a row
      // take the same reference
      if (!fixed && tile_any(tile, !ok || (valid && m_half > m_run + kRescaleThreshold))) {
        if (tile_any(tile, !ok)) {
          ok = false;
          break;
        }
        sm.red[tile][half][R] = m_half;
        tile_sync(tile);
        const float top = fmaxf(sm.red[tile][0][R], sm.red[tile][1][R]);
        float alpha = 1.0f;
        if (top > m_run + kRescaleThreshold) {
          alpha = m_run == -INFINITY ? 0.0f : ex2_approx(m_run - top);
          m_run = top;
        }
        l_run *= alpha;
        if (j > 0 && __any_sync(0xffffffffu, alpha != 1.0f)) {
          // O holds the tile's earlier products (complete: the commit of this S came after them)
          tc_fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            uint32_t o[32];
            tmem_ld32(o_addr + 32 * c, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st32(o_addr + 32 * c, o);
          }
        }
      }
      if (some) {
        const float m_use = (m_run == -INFINITY) ? 0.0f : m_run;
#pragma unroll 1
        for (int c = 0; c < kHalf; c += 32)
          l_run += chunk_exp<kCap>(s_addr + c, s_addr + c / 2, p, u, c, m_use, fixed, valid);
      } else if (warp_live) {
        const uint32_t zeros[16] = {};
        tmem_st16(s_addr, zeros);
        tmem_st16(s_addr + 16, zeros);
      }
      tmem_st_wait();
      tc_fence_before_sync();
      mbar_arrive(&ctl.p_full[tile]);
    }
    if (ok && nt > 0) ok = warp_wait(&ctl.o_full, 0, &ctl.abort);
    if (!ok && lane == 0) {
      if (!ctl.abort) report_status(p.status, kStatusTimeout, 78);
      ctl.abort = 1;
    }

    // ---------------- the rows' results ----------------
    tc_fence_after_sync();
    tile_sync(tile);                      // the last references have been read
    sm.red[tile][half][R] = l_run;
    tile_sync(tile);
    float m = m_run, l = sm.red[tile][0][R] + sm.red[tile][1][R], w = 1.0f, p_self = 0.0f;
    if (fixed) w = follow_sum(m, l);
    if (s_self != -INFINITY) {
      const float m_all = fmaxf(m, s_self);
      const float f = m == -INFINITY ? 0.0f : ex2_approx(m - m_all);
      p_self = ex2_approx(s_self - m_all);
      l = l * f + p_self;
      w *= f;
      m = m_all;
    }
    if (s_self != s_self) l = s_self;   // NaN in the masked-input pair
    const long long orow = rowbase + P;
    const bool split = p.nsplit > 1;
    // 1 / l, once a row; zero where no key was seen
    const float inv = split ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
    if (ok && warp_live) {
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        float o[32] = {};
        if (nt > 0) {
          uint32_t x[32];
          tmem_ld32(o_addr + 32 * c, x);
          tmem_ld_wait(x);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = w == 0.0f ? 0.0f : __uint_as_float(x[e]) * w;
        }
        const int col = half * kHalf + 32 * c;
        if (p_self != 0.0f) add_self(o, p_self, p.v_seedmask + self * kD + col);
        if (valid) store_chunk(p, o, inv, split, ks, orow, col);
        __syncwarp();   // the next chunk is loaded by the whole warp
      }
      if (valid && half == 0) {
        if (split) p.part_ml[static_cast<size_t>(ks) * p.rows + orow] = make_float2(m, l);
        else if (p.lse != nullptr) p.lse[orow] = (m + lg2_approx(l)) * 0.6931471805599453f;
      }
    }
    tc_fence_before_sync();
  }
  __syncthreads();
  if (warp == kPairMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, 512);
  }
}

// ---------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------
// Decoding a KV tile moves 192 KB through shared memory (codes in and out, bf16 in, both products' operands), which
// takes longer than the tile's 32 KB take from HBM, and a Q tile of 128 rows costs the tensor cores the same for one
// row as for 128. For up to kN = 16 or 32 packed rows nothing is decoded: the products are turned over,
//   S^T = K Q^T (128 keys x rows),  O^T += V^T P^T (128 columns x rows),
// and read the e4m3 codes as they are (kind::f8f6f4). Q and P are 8-bit operands there, so each is split in three: a fp16 number of at
// most 9 significant bits is the sum of three e5m2 numbers (e5m2 is the upper byte of fp16: the parts
// are truncations of what the parts before leave, each exact). The parts are columns of their own, 3 kN in all, whose
// products add up in fp32.
//   Q: a row is scaled by a power of two to a maximum of 2^14 .. 2^15 first. bf16 has 8 bits, so the parts are exact down to 2^-23
//      of the row's largest element; what is smaller is cut at e5m2's last bit, 2^-16, below 2^-30 of the largest.
//   P: the V rows' scales belong to the contracted index, so they are taken into the weights: with e_j = x_j - 127 of
//      the V row, P'_j = 2^(s_j + e_j - m), m the row's reference for s_j + e_j, and the sum has 2^(s_j - m) of its
//      own. P' is rounded to 9 bits (off by at most 2^-9 of it; bf16 is by 2^-8) and scaled by 2^12: what is
//      2^-28 of the largest is still held (e5m2's smallest is 2^-16). References take max(e_j, -90) for e_j, so that a row
//      whose largest weight meets a V row far smaller or larger than the others' has a sum within fp32's range; a V row of
//      zeros has e_j = -90. A reference holds V's exponent, so it can change by more than the sum does: from a tile of zeros
//      to one of rows around 2^60 by 150, with a sum of 2^102 before and 2^-48 behind. 2^-150 is no fp32 number, so
//      sums take a change in two halves, within a stream and where streams and parts are added up. (Accumulators need
//      not: where the factor vanishes, what they hold is below 2^-28 of what comes.)
// A softmax thread is a key: its scales are scalars of the thread. The keys' maximum of a row is only taken
// when some score is above the row's reference by more than the threshold (one vote a tile); sums stay with the
// threads until the end. V codes of NaN would reach every row (0 * NaN), so four warps look for them, put zeros in
// their places and report their keys, whose scores become NaN; they report rows of zeros too.
// Streams: alternate KV tiles with sums and an accumulator of their own, merged at the end.
// Roles (480 threads): warps 0-3, 4-7 softmax of the streams; 8-11 NaN codes; 12 products; 13, 14 copies of K, V.
// Tensor memory: S0 | S1 | O0 | O1, 3 kN columns each.
constexpr int kRowsThreads = 480;
constexpr int kScreenWarp = 8, kRowsMmaWarp = 12, kRowsLoadWarp = 13;
constexpr float kRowsThreshold = 2.0f;  // log2 units, of the references' changes
constexpr float kPBits = 12.0f;         // P' carries 2^12 (and is at most 2^14, below fp16's largest)
constexpr int kEvFloor = -90;

// D[tmem] (+)= A[smem] . B[smem] of 8-bit operands
__device__ __forceinline__ void umma_ss_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor for kind::f8f6f4: A e4m3, B e5m2, fp32 accumulation; mn: both are MN-major.
__host__ __device__ constexpr uint32_t idesc_e4m3_e5m2(int M, int N, bool mn) {
  return (1u << 4) | (0u << 7) | (1u << 10) | ((mn ? 3u : 0u) << 15) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

// Barrier of one stream's 128 softmax threads, and with the vote whether any of them says so.
__device__ __forceinline__ void stream_sync(int stream) { asm volatile("bar.sync %0, 128;" ::"r"(2 + stream) : "memory"); }
__device__ __forceinline__ bool stream_any(int stream, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(x ? 1u : 0u), "r"(2 + stream)
      : "memory");
  return r != 0;
}

// fp32 numbers as integers of the same order (no NaN), and back.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

// Two fp16 numbers of at most 9 significant bits as three pairs of e5m2 numbers (in the upper bytes of the halves).
__device__ __forceinline__ void split3(uint32_t x, uint32_t (&part)[3]) {
  part[0] = x & 0xff00ff00u;
  const __half2 r1 = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&part[0]));
  const uint32_t u1 = *reinterpret_cast<const uint32_t*>(&r1);
  part[1] = u1 & 0xff00ff00u;
  const __half2 r2 = __hsub2(r1, *reinterpret_cast<const __half2*>(&part[1]));
  part[2] = *reinterpret_cast<const uint32_t*>(&r2);
}

template <int kN>
struct RowsSmem {
  static constexpr int kStages = 5;
  uint8_t k[kStages][kBN * kD];
  uint8_t v[kStages][kBN * kD];
  uint8_t q[3 * kN * kD];         // parts of Q, [part, row][column]
  uint8_t pt[2][kBN * 128];       // parts of each stream's P^T, [key][part, row], rows of 128 bytes
  uint64_t q_full;
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t v_clean[kStages];      // looked through for NaN codes
  uint64_t s_full[2], p_full[2], o_full, drain;
  uint4 nan_keys[kStages];        // keys with a NaN code in V
  uint4 zero_keys[kStages];       // keys whose V row is zeros
  int4 row[kN];                   // lo, hi, position of a seed row or -1
  float4 fin[kN];                 // weights of the two accumulators and of the masked-input value, 1 / l
  float m[2][kN];                 // per stream: the rows' references m - 12
  float step[2][kN], half[2][kN];    // of the last change: the new reference less the old one, 2 to the opposite of its half
  int unseen[2][kN], any_unseen[2];  // per stream: rows that have seen no key, whose reference is not set
  float red[2][4][kN];            // per stream and warp
  float s_self[kN];
  float2 ml[kN];                  // of a part that the cluster adds up
  float q_scale[kN];              // power of two of a row, times log2(e) / sqrt(d) (capped: 2 log2(e) / (c sqrt(d)))
  int slot[kN];
  uint32_t tmem_base;
  int abort;
  int seq_lo[kMaxShared], seq_hi[kMaxShared];   // keys that some row of a sequence sees
  int lo, hi;                     // keys that some row sees
  int all_lo, all_hi;             // keys that every row sees
};

template <int kN, bool kCap>
__global__ void __launch_bounds__(kRowsThreads, 1)
    attn_prefix8_rows_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                             const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  using Sm = RowsSmem<kN>;
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kStages = Sm::kStages;
  constexpr int kCols = 3 * kN;
  constexpr uint32_t kTmem = kN == 16 ? 256 : 512;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // CTA (ks, group, hkv, b); with parts shared out to the sequences (hkv, group, part), so that those left over come last
  const bool shared_out = p.shares != nullptr;
  int ks, group, hkv, b = 0, slot = 0, nsplit = p.nsplit;
  int rest = static_cast<int>(blockIdx.x);
  if (shared_out) {
    hkv = rest % p.Hkv;
    rest /= p.Hkv;
    group = rest % p.n_groups;
    ks = slot = rest / p.n_groups;
  } else {
    ks = rest % nsplit;
    rest /= nsplit;
    group = rest % p.n_groups;
    rest /= p.n_groups;
    hkv = rest % p.Hkv;
    b = rest / p.Hkv;
  }
  const int n_packed = p.G * p.Lq;
  const int p0 = group * kN;
  int n_rows = min(kN, n_packed - p0);

  if (warp == kRowsMmaWarp) {
    if (lane == 0) {
      mbar_init(&sm.q_full, 256);
      for (int i = 0; i < kStages; ++i) {
        mbar_init(&sm.k_full[i], 1);
        mbar_init(&sm.k_empty[i], 1);
        mbar_init(&sm.v_full[i], 1);
        mbar_init(&sm.v_empty[i], 1);
        mbar_init(&sm.v_clean[i], 128);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], 128);
      }
      mbar_init(&sm.o_full, 1);
      mbar_init(&sm.drain, 1);
      sm.abort = 0;
      sm.any_unseen[0] = sm.any_unseen[1] = 1;
      sm.lo = 0x7fffffff;
      sm.hi = 0;
      sm.all_lo = 0;
      sm.all_hi = p.Lk;
      fence_mbar_init();
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
    }
    __syncwarp();
    tmem_alloc(&sm.tmem_base, kTmem);
    tmem_relinquish();
  }
  if (tid < kN) {
    sm.slot[tid] = kNoSlot;
    sm.s_self[tid] = -INFINITY;
    sm.m[0][tid] = sm.m[1][tid] = 0.0f;
    sm.unseen[0][tid] = sm.unseen[1][tid] = tid < n_rows ? 1 : 0;
  }
  if (tid < kMaxShared) {
    sm.seq_lo[tid] = 0x7fffffff;
    sm.seq_hi[tid] = 0;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = sm.tmem_base;
  griddep_wait();
  griddep_launch_dependents();

  // ---------------- the sequence ----------------
  if (shared_out) {
    for (int i = tid; i < p.B * p.Lq; i += kRowsThreads) {
      const int lo = p.key_lo != nullptr ? max(0, __ldg(p.key_lo + i)) : 0;
      const int hi = p.key_hi != nullptr ? min(p.Lk, __ldg(p.key_hi + i)) : p.Lk;
      if (lo < hi) {
        atomicMin(&sm.seq_lo[i / p.Lq], lo);
        atomicMax(&sm.seq_hi[i / p.Lq], hi);
      }
    }
    __syncthreads();
    const int2 share = share_of(sm.seq_lo, sm.seq_hi, p.B, p.slots);   // of the lane's sequence
    const uint32_t mine = __ballot_sync(0xffffffffu, slot >= share.x && slot < share.x + share.y);
    b = mine != 0 ? __ffs(mine) - 1 : 0;
    ks = slot - __shfl_sync(0xffffffffu, share.x, b);
    nsplit = __shfl_sync(0xffffffffu, share.y, b);
    if (mine == 0) n_rows = 0, ks = nsplit;   // a part that is left over: no rows, no keys
    if (blockIdx.x == 0 && tid < p.B) p.shares[tid] = share;
  }
  const long long rowbase = (static_cast<long long>(b) * p.Hq + hkv * p.G) * p.Lq;
  const size_t mem0 = (static_cast<size_t>(b) * p.Hkv + hkv) * p.Lk;
  // the part's first row, less the first row of what it is a part of
  const long long part0 = shared_out ? (static_cast<long long>(slot) - b) * p.Hq * p.Lq : ks * p.rows;

  // ---------------- the rows ----------------
  const bool ranges = p.key_lo != nullptr || p.key_hi != nullptr;
  const int r0 = p.Lq <= kN ? 0 : p0 % p.Lq;   // the rows stand at up to kN positions: r itself, or r - r0 around Lq
  if (p.n_seeds > 0) {
    const int32_t* seeds = p.seed_idx + static_cast<size_t>(b) * p.n_seeds;
    for (int s = tid; s < p.n_seeds; s += kRowsThreads) {
      const int at = __ldg(seeds + s) - p.q0;
      if (at < 0 || at >= p.Lq) continue;
      const int i = at >= r0 ? at - r0 : at - r0 + p.Lq;
      if (i < kN) atomicMin(&sm.slot[i], s);
    }
    __syncthreads();
  }
  if (ranges || p.n_seeds > 0) {
    int my_slot = kNoSlot;
    if (tid < kN) {
      int lo = 0, hi = p.Lk, at = -1;
      if (tid < n_rows) {
        const int r = (p0 + tid) % p.Lq;
        const size_t i = static_cast<size_t>(b) * p.Lq + r;
        if (p.key_lo != nullptr) lo = max(0, __ldg(p.key_lo + i));
        if (p.key_hi != nullptr) hi = min(p.Lk, __ldg(p.key_hi + i));
        if (p.n_seeds > 0) {
          my_slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq];
          if (my_slot != kNoSlot) at = p.q0 + r;
        }
        if (ranges) {
          if (lo < hi) {
            atomicMin(&sm.lo, lo);
            atomicMax(&sm.hi, hi);
          }
          atomicMax(&sm.all_lo, lo);
          atomicMin(&sm.all_hi, hi);
        }
      }
      sm.row[tid] = make_int4(lo, hi, at, 0);
    }
    __syncthreads();
    // the slots by row, now that they are read by position
    if (tid < kN) sm.slot[tid] = my_slot;
    __syncthreads();
  } else if (tid < kN) {
    sm.row[tid] = make_int4(0, p.Lk, -1, 0);   // read by the softmax warps, after their barrier
  }
  Part part = ranges ? part_of(sm.lo, sm.hi, ks, nsplit) : part_of(0, p.Lk, ks, nsplit);
  if (ks >= nsplit) part.nt = 0;
  const int j0 = part.j0, nt = part.nt;

  if (warp >= kRowsMmaWarp) {
    if ((warp == kRowsLoadWarp || warp == kRowsLoadWarp + 1) && lane == 0 && nt > 0) {
      // ---------------- copies ----------------
      const int which = warp - kRowsLoadWarp;
      const CUtensorMap* tm = which ? &tm_v : &tm_k;
      uint64_t* const full = which ? sm.v_full : sm.k_full;
      uint64_t* const empty = which ? sm.v_empty : sm.k_empty;
      bool ok = true;
      int j = 0;
      for (; j < nt; ++j) {
        const int st = j % kStages;
        if (j >= kStages) ok = mbar_wait(&empty[st], (j / kStages - 1) & 1, &sm.abort);
        if (!ok) break;
        mbar_arrive_expect_tx(&full[st], kBN * kD);
        tma_load_4d(which ? sm.v[st] : sm.k[st], tm, &full[st], 0, (j0 + j) * kBN, hkv, b);   // zeros past the memory
      }
      if (!ok) {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 70);
        sm.abort = 1;
      }
      // every copy lands before the CTA's shared memory is released, whatever the other roles did
      for (int f = max(0, j - kStages); f < j; ++f) mbar_wait(&full[f % kStages], (f / kStages) & 1, nullptr);
    } else if (warp == kRowsMmaWarp && lane == 0 && nt > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_s = idesc_e4m3_e5m2(kBN, kCols, false);
      constexpr uint32_t id_o = idesc_e4m3_e5m2(kD, kCols, true);
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q), 16, 1024);
      const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
      const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), 16, 1024);
      const uint64_t dp = sdesc_sw128(smem_u32(sm.pt[0]), 16, 1024);
      constexpr uint32_t kStageDesc = (kBN * kD) >> 4;
      // descriptors are added up in their lower words (4 x 131072 keys, 32 / 8 heads: 187 -> 182.6 us)
      const uint32_t q_lo = static_cast<uint32_t>(dq), k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv),
                     p_lo = static_cast<uint32_t>(dp), hi = static_cast<uint32_t>(dq >> 32);   // (all four have the same upper words)
      const auto desc = [&](uint32_t lo) { return (static_cast<uint64_t>(hi) << 32) | lo; };
      // S^T[s] = K(tile j) . Q^T
      auto issue_s = [&](int j) {
        const int s = j & 1, st = j % kStages;
        const uint32_t k = k_lo + st * kStageDesc;
#pragma unroll
        for (int kk = 0; kk < kD / 32; ++kk)
          umma_ss_f8(tbase + s * kCols, desc(k + ((kk * 32) >> 4)), desc(q_lo + ((kk * 32) >> 4)), id_s, kk > 0 ? 1u : 0u);
        umma_commit(&sm.s_full[s]);
        umma_commit(&sm.k_empty[st]);
      };
      // O^T[s] (+)= V(tile j)^T . P[s]^T
      auto issue_o = [&](int j) {
        const int s = j & 1, st = j % kStages;
        const uint32_t v = v_lo + st * kStageDesc, pt = p_lo + s * ((kBN * 128) >> 4);
#pragma unroll
        for (int kk = 0; kk < kBN / 32; ++kk)
          umma_ss_f8(tbase + (2 + s) * kCols, desc(v + ((kk * 32 * kD) >> 4)), desc(pt + ((kk * 32 * 128) >> 4)), id_o,
                     (j > 1 || kk > 0) ? 1u : 0u);
        umma_commit(&sm.v_empty[st]);
      };
      auto wait = [&](uint64_t* bar, int phase) {
        const bool ok = mbar_wait(bar, phase & 1, &sm.abort);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      bool ok = wait(&sm.q_full, 0);
      for (int j = 0; j < 2 && j < nt && ok; ++j) {
        ok = wait(&sm.k_full[j], 0);
        if (ok) issue_s(j);
      }
      for (int j = 0; j < nt && ok; ++j) {
        ok = wait(&sm.v_clean[j % kStages], j / kStages) && wait(&sm.p_full[j & 1], j >> 1);
        if (!ok) break;
        issue_o(j);
        if (j + 2 < nt) {
          ok = wait(&sm.k_full[(j + 2) % kStages], (j + 2) / kStages);
          if (ok) issue_s(j + 2);
        }
      }
      if (ok) {
        umma_commit(&sm.o_full);
      } else {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 74);
        sm.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&sm.drain);
      mbar_wait(&sm.drain, 0, nullptr);
    }
    if (p.joined) join_pass();
  } else if (warp >= kScreenWarp) {
    // ---------------- NaN codes of V (thread = key; the swizzle moves no byte out of its row) ----------------
    const int key = tid - kScreenWarp * 32;
    bool ok = true;
    for (int j = 0; j < nt; ++j) {
      const int st = j % kStages;
      ok = warp_wait(&sm.v_full[st], (j / kStages) & 1, &sm.abort);
      if (!ok) break;
      const uint32_t row = smem_u32(sm.v[st]) + key * kD;
      uint32_t hit = 0, any = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 c = lds128(row + ((i ^ (key & 7)) << 4));
        any |= c.x | c.y | c.z | c.w;
        hit |= ((c.x & 0x7f7f7f7fu) + 0x01010101u) | ((c.y & 0x7f7f7f7fu) + 0x01010101u) |
               ((c.z & 0x7f7f7f7fu) + 0x01010101u) | ((c.w & 0x7f7f7f7fu) + 0x01010101u);
      }
      const bool bad = (hit & 0x80808080u) != 0;
      const uint32_t nans = __ballot_sync(0xffffffffu, bad), zeros = __ballot_sync(0xffffffffu, (any & 0x7f7f7f7fu) == 0);
      if (bad) {
#pragma unroll 1
        for (int i = 0; i < 8; ++i) sts128(row + 16 * i, 0, 0, 0, 0);
      }
      if (lane == 0) {
        reinterpret_cast<uint32_t*>(&sm.nan_keys[st])[key >> 5] = nans;
        reinterpret_cast<uint32_t*>(&sm.zero_keys[st])[key >> 5] = zeros;
      }
      fence_proxy_async_smem();
      mbar_arrive(&sm.v_clean[st]);
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 72);
      sm.abort = 1;
    }
    if (p.joined) join_pass();
  } else {
    // ---------------- softmax (thread = key of a KV tile) ----------------
    const int stream = warp >> 2, key = tid & (kBN - 1), w4 = warp & 3;
    const size_t masked0 = (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds;   // masked-input rows of this KV head
    // the exponent bytes of the thread's first two tiles are on their way while Q is made ready
    const uint8_t* kx = p.k_exp + mem0 + static_cast<size_t>(j0) * kBN + key;
    const uint8_t* vx = p.v_exp + mem0 + static_cast<size_t>(j0) * kBN + key;
    const int left = p.Lk - j0 * kBN - key;   // the thread's key of tile j is in the memory if j * kBN < left
    uint32_t xk[2], xv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = (stream + 2 * i) * kBN;
      const bool in = stream + 2 * i < nt && at < left;
      xk[i] = in ? __ldg(kx + at) : 127u;
      xv[i] = in ? __ldg(vx + at) : 127u;
    }
    // parts of Q, a warp a row: lane's columns 4 lane .. 4 lane + 3
    for (int n = warp; n < kN; n += 8) {
      uint2 a = make_uint2(0, 0);
      if (n < n_rows) a = __ldg(reinterpret_cast<const uint2*>(p.q + (rowbase + p0 + n) * kD) + lane);
      const float f[4] = {__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u), __uint_as_float(a.y << 16),
                          __uint_as_float(a.y & 0xffff0000u)};
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
      top = __reduce_max_sync(0xffffffffu, top);
      // a maximum of 2^e .. 2^(e + 1) goes to 2^14 .. 2^15; e held to -112 .. 127 (subnormal rows lose their last bits)
      const int e = min(max(static_cast<int>(top >> 23) - 127, -112), 127);
      const float up = __uint_as_float(static_cast<uint32_t>(14 - e + 127) << 23);
      const bool bad = (top >> 23) == 255;   // a row with an element that is not finite has NaN scores
      uint32_t part0[3], part1[3];
      const __half2 h0 = __floats2half2_rn(bad ? 0.0f : f[0] * up, bad ? 0.0f : f[1] * up);
      const __half2 h1 = __floats2half2_rn(bad ? 0.0f : f[2] * up, bad ? 0.0f : f[3] * up);
      split3(*reinterpret_cast<const uint32_t*>(&h0), part0);
      split3(*reinterpret_cast<const uint32_t*>(&h1), part1);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int row = i * kN + n;
        const uint32_t four = __byte_perm(part0[i], part1[i], 0x7531);   // the upper bytes of four halves
        *reinterpret_cast<uint32_t*>(sm.q + row * kD + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4) = four;
      }
      if (lane == 0)
        sm.q_scale[n] = bad ? __uint_as_float(0x7fc00000u)
                            : __uint_as_float(static_cast<uint32_t>(e - 14 + 127) << 23) * (kCap ? p.cap_in : p.scale_log2);
    }
    fence_proxy_async_smem();
    mbar_arrive(&sm.q_full);
    // the seed rows' own scores (log2 units), in the first part alone: a warp a row, four columns a lane
    if (p.n_seeds > 0 && ks == 0) {
      for (int n = warp; n < n_rows; n += 8) {
        const int4 info = sm.row[n];
        if (info.z < 0 || info.z < info.x || info.z >= info.y) continue;
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(p.q + (rowbase + p0 + n) * kD) + lane);
        const uint2 c = __ldg(reinterpret_cast<const uint2*>(p.k_seedmask + (masked0 + sm.slot[n]) * kD) + lane);
        float dot = __uint_as_float(a.x << 16) * __uint_as_float(c.x << 16);
        dot = fmaf(__uint_as_float(a.x & 0xffff0000u), __uint_as_float(c.x & 0xffff0000u), dot);
        dot = fmaf(__uint_as_float(a.y << 16), __uint_as_float(c.y << 16), dot);
        dot = fmaf(__uint_as_float(a.y & 0xffff0000u), __uint_as_float(c.y & 0xffff0000u), dot);
        for (int d = 16; d >= 1; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
        if (lane == 0) sm.s_self[n] = kCap ? capped(dot, p.cap_in, p.cap_log2) : dot * p.scale_log2;
      }
    }
    softmax_sync();   // q_scale and row are written
    const uint32_t quad = tbase + (static_cast<uint32_t>(w4 * 32) << 16);
    const uint32_t s_addr = quad + stream * kCols, o_addr = quad + (2 + stream) * kCols;
    const float* m = sm.m[stream];
    const uint32_t pt = smem_u32(sm.pt[stream]) + key * 128;
    const uint32_t sw = static_cast<uint32_t>(key & 7) << 4;
    const int all_lo = sm.all_lo, all_hi = sm.all_hi;
    float l[kN];
#pragma unroll
    for (int n = 0; n < kN; ++n) l[n] = 0.0f;
    bool ok = true;
    int i = 0;
    for (int j = stream; j < nt; j += 2, ++i) {
      // (the asm keeps the bytes' loads from being waited for before this tile)
      asm volatile("" : "+r"(xk[0]), "+r"(xv[0]));
      const int k_byte = static_cast<int>(xk[0]), v_byte = static_cast<int>(xv[0]);
      xk[0] = xk[1], xv[0] = xv[1];
      if (j + 4 < nt && (j + 4) * kBN < left) {
        xk[1] = __ldg(kx + (j + 4) * kBN);
        xv[1] = __ldg(vx + (j + 4) * kBN);
      }
      const int st = j % kStages;
      ok = warp_wait(&sm.s_full[stream], i & 1, &sm.abort) && warp_wait(&sm.v_clean[st], (j / kStages) & 1, &sm.abort);
      float t[kN];        // s_j + e_j - m + 12, in log2 units
      bool over = !ok;    // a warp whose wait gave up votes all the same: the stream's barriers take 128 threads
      // bytes above 246 count as NaN (cover_kv8_write writes none but 255)
      // a V row of zeros has the smallest exponent, whatever its byte: however large its key's weight, it leaves the
      // reference to the others
      const bool zero_v = ok && ((reinterpret_cast<const uint32_t*>(&sm.zero_keys[st])[key >> 5] >> (key & 31)) & 1u);
      const float e_v = static_cast<float>(zero_v ? kEvFloor : v_byte - 127);
      const float lift = fmaxf(e_v, static_cast<float>(kEvFloor)) - e_v;
      if (ok) {
        tc_fence_after_sync();
        const bool nan_key = v_byte > kExpMax || k_byte > kExpMax ||
                             ((reinterpret_cast<const uint32_t*>(&sm.nan_keys[st])[key >> 5] >> (key & 31)) & 1u);
        const float k_scale = nan_key ? __uint_as_float(0x7fc00000u) : e4m3_scale(k_byte);
#pragma unroll
        for (int c = 0; c < kN; c += 16) {
          uint32_t x[3][16];
#pragma unroll
          for (int h = 0; h < 3; ++h) tmem_ld16(s_addr + h * kN + c, x[h]);
#pragma unroll
          for (int h = 0; h < 3; ++h) tmem_ld_wait16(x[h]);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float sum = (__uint_as_float(x[2][e]) + __uint_as_float(x[1][e])) + __uint_as_float(x[0][e]);
            const float f = k_scale * sm.q_scale[c + e];
            t[c + e] = (kCap ? capped(sum, f, p.cap_log2) + e_v : fmaf(sum, f, e_v)) - m[c + e];
          }
        }
        // keys that some row does not see, among them a seed row's own cached column
        const int key0 = (j0 + j) * kBN, at = key0 + key;
        if (key0 < all_lo || key0 + kBN > all_hi ||
            (p.n_seeds > 0 && key0 < p.q0 + p.Lq && key0 + kBN > p.q0)) {
#pragma unroll
          for (int n = 0; n < kN; ++n) {
            const int4 info = sm.row[n];
            if (at < info.x || at >= info.y || at == info.z) t[n] = -INFINITY;
          }
        }
        const float margin = kRowsThreshold + kPBits - lift;
#pragma unroll
        for (int n = 0; n < kN; ++n) over |= t[n] > margin;
        over |= sm.any_unseen[stream] != 0;
        __syncwarp();
      }
      if (stream_any(stream, over)) {
        if (stream_any(stream, !ok)) {
          ok = false;
          break;
        }
        // new references: the rows' maxima where they are above the old ones by more than the threshold
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          const int top = __reduce_max_sync(0xffffffffu, ordered(t[n] == t[n] ? t[n] + lift : -INFINITY));
          if (lane == (n & 31)) sm.red[stream][w4][n] = from_ordered(top);
        }
        stream_sync(stream);
        if (key < kN) {
          const float up = fmaxf(fmaxf(sm.red[stream][0][key], sm.red[stream][1][key]),
                                 fmaxf(sm.red[stream][2][key], sm.red[stream][3][key])) - kPBits;
          // a row's first keys set its reference, wherever they lie
          const bool first = sm.unseen[stream][key] != 0 && up > -INFINITY;
          const float step = first || up > kRowsThreshold ? up : 0.0f;
          sm.step[stream][key] = step;
          sm.half[stream][key] = first ? 0.0f : ex2_approx(-0.5f * step);
          sm.m[stream][key] = m[key] + step;
          if (first) sm.unseen[stream][key] = 0;
          const uint32_t mask = kN == 32 ? 0xffffffffu : 0xffffu;
          const uint32_t still = __ballot_sync(mask, sm.unseen[stream][key] != 0);
          if (key == 0) sm.any_unseen[stream] = still != 0 ? 1 : 0;
        }
        stream_sync(stream);
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          const float half = sm.half[stream][n];
          t[n] -= sm.step[stream][n];
          l[n] = l[n] * half * half;
        }
        if (i > 0) {
          // O holds the stream's earlier products (complete: the commit of this S came after them)
#pragma unroll
          for (int c = 0; c < kCols; c += 16) {
            uint32_t o[16];
            tmem_ld16(o_addr + c, o);
            tmem_ld_wait16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float half = sm.half[stream][c % kN + e];
              o[e] = __float_as_uint(__uint_as_float(o[e]) * (half * half));
            }
            tmem_st16(o_addr + c, o);
          }
          tmem_st_wait();
        }
      }
#pragma unroll
      for (int c = 0; c < kN; c += 16) {
        uint32_t out[3][4];   // parts of 16 rows
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          uint32_t parts[2][3];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int n = c + 4 * q4 + 2 * h;
            const float e0 = ex2_approx(t[n]), e1 = ex2_approx(t[n + 1]);
            l[n] += ex2_approx(t[n] - e_v);
            l[n + 1] += ex2_approx(t[n + 1] - e_v);
            // to 9 significant bits, half up: P' is at most 2^14, so that no carry leaves a half
            const __half2 x = __floats2half2_rn(e0, e1);
            split3((*reinterpret_cast<const uint32_t*>(&x) + 0x00020002u) & 0xfffcfffcu, parts[h]);
          }
#pragma unroll
          for (int i3 = 0; i3 < 3; ++i3) out[i3][q4] = __byte_perm(parts[0][i3], parts[1][i3], 0x7531);
        }
#pragma unroll
        for (int i3 = 0; i3 < 3; ++i3)
          sts128(pt + ((static_cast<uint32_t>(i3 * kN + c)) ^ sw), out[i3][0], out[i3][1], out[i3][2], out[i3][3]);
      }
      fence_proxy_async_smem();
      tc_fence_before_sync();
      mbar_arrive(&sm.p_full[stream]);
    }
    if (ok && nt > 0) ok = warp_wait(&sm.o_full, 0, &sm.abort);
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 75);
      sm.abort = 1;
    }

    // ---------------- the rows' results ----------------
    tc_fence_after_sync();
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      float x = l[n];
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      if (lane == (n & 31)) sm.red[stream][w4][n] = x;
    }
    softmax_sync();
    const bool split = shared_out || p.nsplit > 1;
    const uint32_t staged = smem_u32(sm.k[0]);   // every product is complete: K is not read any more
    if (ok && tid < n_rows) {
      const int n = tid;
      const long long orow = rowbase + p0 + n;
      const float s_self = sm.s_self[n];
      float l2[2];
      for (int s = 0; s < 2; ++s) l2[s] = (sm.red[s][0][n] + sm.red[s][1][n]) + (sm.red[s][2][n] + sm.red[s][3][n]);
      const float m0 = sm.unseen[0][n] ? -INFINITY : sm.m[0][n], m1 = sm.unseen[1][n] ? -INFINITY : sm.m[1][n];
      const float top = fmaxf(fmaxf(m0, m1), s_self);
      // halves of the streams' factors: a factor itself may be no fp32 number where its sum is large
      const float h0 = m0 == -INFINITY ? 0.0f : ex2_approx(0.5f * (m0 - top)), h1 = m1 == -INFINITY ? 0.0f : ex2_approx(0.5f * (m1 - top));
      const float p_self = s_self == -INFINITY ? 0.0f : ex2_approx(s_self - top);
      // (NaN scores leave the references alone: they are in the sums)
      float sum = fmaf(h0 * l2[0], h0, fmaf(h1 * l2[1], h1, p_self));
      if (l2[0] != l2[0] || l2[1] != l2[1]) sum = l2[0] + l2[1];
      if (s_self != s_self) sum = s_self;
      sm.fin[n] = make_float4(h0 * h0, h1 * h1, p_self, split ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum);
      if (p.joined) sm.ml[n] = make_float2(top, sum);
      else if (split) p.part_ml[part0 + orow] = make_float2(top, sum);
      else if (p.lse != nullptr) p.lse[orow] = (top + lg2_approx(sum)) * 0.6931471805599453f;
    }
    softmax_sync();
    // thread = output column; the streams' warps take 16 rows in turn
    const int col = key;
    for (int c = 16 * stream; c < n_rows; c += 32) {
      if (!ok) break;
      float o0[16] = {}, o1[16] = {};
      if (nt > 0) {
#pragma unroll
        for (int h = 2; h >= 0; --h) {
          uint32_t x[16];
          tmem_ld16(quad + 2 * kCols + h * kN + c, x);
          tmem_ld_wait16(x);
#pragma unroll
          for (int e = 0; e < 16; ++e) o0[e] += __uint_as_float(x[e]);
          if (nt > 1) {
            tmem_ld16(quad + 3 * kCols + h * kN + c, x);
            tmem_ld_wait16(x);
#pragma unroll
            for (int e = 0; e < 16; ++e) o1[e] += __uint_as_float(x[e]);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int n = c + e;
        if (n < n_rows) {
          const float4 f = sm.fin[n];
          float o = f.x == 0.0f ? 0.0f : o0[e] * f.x;
          if (f.y != 0.0f) o = fmaf(o1[e], f.y, o);
          if (f.z != 0.0f) o = fmaf(f.z, __bfloat162float(p.v_seedmask[(masked0 + sm.slot[n]) * kD + col]), o);
          const long long orow = rowbase + p0 + n;
          if (p.joined) sts32(staged + staged_at(n, col >> 2) + 4 * (col & 3), __float_as_uint(o));
          else if (split) p.part_o[(part0 + orow) * kD + col] = o;
          else p.out[orow * kD + col] = __float2bfloat16_rn(o * f.w);
        }
      }
      __syncwarp();
    }
    tc_fence_before_sync();
    if (p.joined) join_parts<false>(p, staged, smem_u32(sm.ml), n_rows, rowbase + p0, ks);
  }
  __syncthreads();
  if (warp == kRowsMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, kTmem);
  }
}

// Combines the parts of every row: one warp a row, four columns a lane.
constexpr int kCombineWarps = 4;
__global__ void __launch_bounds__(kCombineWarps * 32)
    attn_prefix8_combine_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, int nsplit,
                                const int2* shares, long long seq_rows, long long rows, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kCombineWarps + (threadIdx.x >> 5);
  if (row >= rows) return;
  long long first = row, step = rows;   // the row in its first part, and from part to part
  if (shares != nullptr) {
    const long long b = row / seq_rows;
    const int2 share = shares[b];
    first = (share.x - b) * seq_rows + row;
    nsplit = share.y;
    step = seq_rows;
  }
  float m = -INFINITY;
  for (int j = lane; j < nsplit; j += 32) m = fmaxf(m, part_ml[first + j * step].x);
  for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  const float m_use = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int j = 0; j < nsplit; ++j) {
    const float2 ml = part_ml[first + j * step];
    const float4 o = *reinterpret_cast<const float4*>(part_o + (first + j * step) * kD + 4 * lane);
    const float half = ml.x == -INFINITY ? 0.0f : ex2_approx(0.5f * (ml.x - m_use)), w = half * half;
    l = fmaf(half * ml.y, half, l);
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

// kDecodedPairs: pairs of Q tiles over a memory that a pass of its own decodes first; kReadBack: cover_attn_fwd_prefix's
// kernels over such a memory, where every row sees every key and scores are not capped
enum Mode { kRows16, kRows32, kTile, kDecodedPairs, kReadBack };
constexpr int kModes = 5;
constexpr int kModeRows[kModes] = {16, 32, kBM, 2 * kBM, 1};   // packed rows of a CTA

// Capped scores lie in [-C, C], C = cap log2(e). For C <= 75 (caps up to 52) every row takes the same reference, C - 45 or
// 0, and no maxima are looked for: the weights lie in [2^(45 - 2 C), 2^45], at least 2^-105. (Caps below 2^-10 would put powers
// of 1 / cap beyond fp32's largest number.)
float fixed_reference(float cap_log2) {
  return cap_log2 >= 1.0f / 1024.0f && cap_log2 <= 75.0f ? fmaxf(0.0f, cap_log2 - 45.0f) : -INFINITY;
}
// The bytes of V rows that such a reference serves: L keys of the largest weight and the largest code (below 2^9) stay below
// 2^126, and the smallest weight times the smallest code (2^-9) is not below 2^-126. Cap 30 over 8192 keys: 53 .. 188, values up
// to 2^70; cap 50: 110 .. 187, rows whose largest element is above 0.002. A CTA one of whose V rows has another byte looks
// for maxima.
void fixed_bytes(float cap_log2, float cap_ref, int L, uint32_t* lo, uint32_t* hi) {
  *lo = static_cast<uint32_t>(std::max(0.0f, std::ceil(10.0f + cap_log2 + cap_ref)));
  *hi = static_cast<uint32_t>(std::floor(127.0f + 126.0f - 9.0f - (cap_log2 - cap_ref) - std::ceil(std::log2(static_cast<float>(L)))));
}

// Whether the parts of a batch with key ranges can be shared out to its sequences (every CTA looks through the ranges).
bool shares_out(int B, int Lq) { return B > 1 && B <= kMaxShared && static_cast<long long>(B) * Lq <= 2048; }

struct Plan {
  Mode mode;
  int n_groups, nsplit;
  bool joined;   // the parts' CTAs are clusters
  int slots;     // parts of a KV head shared out to the sequences (0: nsplit each)
  double us;
};

// Resident clusters of 1 .. 8 CTAs, one CTA an SM, that the prediction for cover_attn_fwd_prefix's kernels goes by.
constexpr int kClusters[8] = {152, 76, 48, 36, 28, 24, 20, 18};
// The same for the parts joined in a cluster: at least so many on every GPU measured (they differ: 15 or 18 of 8 CTAs),
// and calls of 28 clusters of 5 took two turns where 28 fitted.
constexpr int kJoinedClusters[kMaxJoined] = {152, 76, 46, 36, 24, 20, 14, 14};

// The kernel and the parts of the keys. plain: no key ranges, no cap.
//
// Predicted microseconds, fitted to 631 calls back to back on GB300 (24 windows of 1 to 1024 rows over 300 to 20000
// keys, batches of 1 to 16, 1 to 64 parts; off by 4 to 9 % in the mean, at most 40 %): a base, and for every wave of one
// CTA an SM a start and a time per KV tile; where the keys are in parts, the second kernel's start, its walk over the
// parts, and the parts' rows, or, joined in a cluster, the cluster's barriers and the rows that a CTA finishes. Decoding a
// memory takes 1e-4 us a row. In each of the 24 the call's choice took at most 5 % longer than the fastest of all
// kernels and parts (one of them 9 %, where two launches would be faster on the device and slower on the host). Joined against added up by a second kernel, each with its best parts: 8.3 against 10.0 us (1 x 28 / 4
// heads, 1 x 777), 10.3 / 11.9 (1 x 4000), 12.9 / 15.1 (1 x 32 / 8, 128 x 1024), 22.7 / 24.8 (4 x 16 / 2, 64 x 4096);
// the second kernel's where more than 8 parts pay: 22.5 / 19.5 (1 x 28 / 4, 32 x 8192).
struct ModeCost {
  double base, wave, tile, combine, row, join, join_row;
};
constexpr ModeCost kCosts[kReadBack] = {
    {2.2, 4.5, 0.72, 0.8, 6.4e-4, 0.8, 0.07}, {2.4, 6.0, 0.92, 0.8, 4.8e-4, 0.6, 0.13},
    {3.0, 4.1, 1.34, 1.5, 2.5e-4, 2.0, 0.036}, {5.0, 3.5, 1.60, 2.4, 1.9e-4, 0.0, 0.0}};
constexpr double kFill = 0.75, kShareUs = 1.0;
constexpr double kPartUs = 0.15, kDecodeRowUs = 1.0e-4, kDecodeUs = 1.8;

Plan plan_of(int B, int Hq, int Hkv, int Lq, int L, bool plain, bool ranges) {
  Plan best{};
  const long long packed = static_cast<long long>(Hq / Hkv) * Lq;
  const double rows = static_cast<double>(B) * Hq * Lq, decode_us = kDecodeRowUs * B * Hkv * L;
  const int nkv = (L + kBN - 1) / kBN;
  for (int mode = 0; mode < kReadBack; ++mode) {
    if (mode > 0 && kModeRows[mode - 1] >= packed) continue;   // a smaller one holds all rows
    const ModeCost& k = kCosts[mode];
    const long long groups = (packed + kModeRows[mode] - 1) / kModeRows[mode];
    const long long units = groups * Hkv * B;
    for (int ns = 1; ns <= nkv && ns <= kMaxParts; ++ns) {
      const long long waves = (units * ns + kSms - 1) / kSms;
      const int tiles = (nkv + ns - 1) / ns;
      const double us = k.base + waves * (k.wave + k.tile * tiles) + (mode == kDecodedPairs ? decode_us : 0.0) +
                        (ns > 1 ? k.combine + kPartUs * ns + k.row * rows * ns : 0.0);
      if (best.nsplit == 0 || us < best.us) best = Plan{static_cast<Mode>(mode), static_cast<int>(groups), ns, false, 0, us};
      if (mode != kDecodedPairs && ns > 1 && ns <= kMaxJoined) {
        const long long turns = (units + kJoinedClusters[ns - 1] - 1) / kJoinedClusters[ns - 1];
        const double own_rows = std::ceil(std::min<double>(packed, kModeRows[mode]) / ns);
        const double join_us = k.base + turns * (k.wave + k.tile * tiles + k.join + k.join_row * own_rows);
        if (join_us < best.us) best = Plan{static_cast<Mode>(mode), static_cast<int>(groups), ns, true, 0, join_us};
      }
      if (units * ns > 8 * kSms) break;
    }
    if (ranges && mode <= kRows32 && shares_out(B, Lq)) {
      // one wave of parts, of kFill of the memories' tiles. Rounded to whole parts the sequences' shares are fair from three
      // parts a sequence on: 4 x 32 / 8 heads over 131072, 79828, 102273 and 0 keys 117 us (9 parts each 145; with all
      // four full 205 and 197), 8 x 28 / 4 over 15681 to 40000 keys 51 (joined in fours 72), but 16 x 32 / 8 over 2786
      // to 8192 keys 59 (57 without parts). Two waves of parts: 132, 64, 53.
      const long long slots = std::min<long long>(kSms / (groups * Hkv), static_cast<long long>(B) * kMaxParts);
      const double tiles = std::ceil(kFill * B * nkv / std::max<long long>(slots, 1)) + 1, parts = static_cast<double>(slots) / B;
      const double us = k.base + kShareUs + k.wave + k.tile * tiles + k.combine + kPartUs * parts + k.row * rows * parts;
      if (slots >= 3 * B && us < best.us) best = Plan{static_cast<Mode>(mode), static_cast<int>(groups), 1, false, static_cast<int>(slots), us};
    }
  }
  if (plain) {
    AttnArgs a{};
    a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.L = L, a.D = kD, a.Lq = Lq, a.q0 = 0;
    double us = 4.0 + 0.91 * window_square_us(a, kSms);   // as measured behind the decoding pass (250 us where it says 272, 14 for 12)
    const WindowChoice c = window_gqa_model(a, kSms, kClusters);
    if (c.packed) us = std::min(us, c.packed_us);
    us += kDecodeUs + decode_us;
    if (us < best.us) best = Plan{kReadBack, 1, 1, false, 0, us};
  }
  return best;
}

using RowsKernel = void (*)(const CUtensorMap, const CUtensorMap, const Params);
using TileKernel = void (*)(const CUtensorMap, const Params);
using PairKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const Params);
constexpr TileKernel kTileKernels[2] = {attn_prefix8_tile_kernel<false>, attn_prefix8_tile_kernel<true>};
constexpr PairKernel kPairKernels[2] = {attn_prefix8_pairs_kernel<false>, attn_prefix8_pairs_kernel<true>};
constexpr size_t kPairSmemBytes = sizeof(PairSmem) + 1024;
static_assert(kPairSmemBytes <= 227 * 1024, "shared memory of a CTA");
constexpr RowsKernel kRowsKernels[2][2] = {{attn_prefix8_rows_kernel<16, false>, attn_prefix8_rows_kernel<16, true>},
                                           {attn_prefix8_rows_kernel<32, false>, attn_prefix8_rows_kernel<32, true>}};
constexpr size_t kRowsSmemBytes[2] = {sizeof(RowsSmem<16>) + 1024, sizeof(RowsSmem<32>) + 1024};
static_assert(kRowsSmemBytes[0] <= 227 * 1024 && kRowsSmemBytes[1] <= 227 * 1024, "shared memory of a CTA");

// The workspace: the parts' accumulators and sums, or the decoded K and V (both where both are needed).
size_t decoded_bytes(const Plan& plan, int B, int Hkv, int L) {
  return plan.mode >= kDecodedPairs ? static_cast<size_t>(B) * Hkv * L * kD * 2 : 0;   // of K, and of V
}
// rows of all parts
size_t part_rows(const Plan& plan, int B, int Hq, int Lq) {
  if (plan.slots > 0) return static_cast<size_t>(plan.slots + B) * Hq * Lq;
  return plan.nsplit <= 1 || plan.joined ? 0 : static_cast<size_t>(B) * Hq * Lq * plan.nsplit;
}
size_t plan_bytes(const Plan& plan, int B, int Hq, int Hkv, int Lq, int L) {
  const size_t parts = part_rows(plan, B, Hq, Lq) * (kD * sizeof(float) + sizeof(float2));
  return 2 * decoded_bytes(plan, B, Hkv, L) + (plan.slots > 0 ? parts + kMaxShared * sizeof(int2) : (parts + 15) & ~size_t{15});
}

// The keys' parts as one number: 1 .. 64 for the second kernel, -2 .. -8 joined, kSharedCode + the parts shared out.
int parts_code(const Plan& p) { return p.slots > 0 ? kAttn8SharedCode + p.slots : p.joined ? -p.nsplit : p.nsplit; }
void set_parts(Plan& p, int code) {
  p.slots = code > kAttn8SharedCode ? code - kAttn8SharedCode : 0;
  p.joined = code < 0;
  p.nsplit = p.slots > 0 ? 1 : std::abs(code);
}

}  // namespace

size_t attn_prefix8_workspace_bytes(int B, int Hq, int Hkv, int Lq, int L) {
  size_t most = 0;
  for (int i = 0; i < 3; ++i)
    most = std::max(most, plan_bytes(plan_of(B, Hq, Hkv, Lq, L, i == 0, i == 1), B, Hq, Hkv, Lq, L));
  return most;
}

void attn_prefix8_plan(int B, int Hq, int Hkv, int Lq, int L, bool plain, bool ranges, int* choice, double* us) {
  const Plan p = plan_of(B, Hq, Hkv, Lq, L, plain, ranges);
  choice[0] = p.mode;
  choice[1] = p.n_groups;
  choice[2] = parts_code(p);
  *us = p.us;
}

size_t attn_prefix8_mode_bytes(int B, int Hq, int Hkv, int Lq, int L, int mode, int parts) {
  Plan p{static_cast<Mode>(mode), 1, 1, false, 0, 0.0};
  set_parts(p, parts);
  return plan_bytes(p, B, Hq, Hkv, Lq, L);
}

int launch_attn_prefix8(const Attn8Args& a, int* status, cudaStream_t stream) {
  const long long rows = static_cast<long long>(a.B) * a.Hq * a.Lq;
  if (rows + 2 * kBM > 0x7fffffffLL) return -2;
  const bool ranges = a.key_lo != nullptr || a.key_hi != nullptr;
  Plan plan = plan_of(a.B, a.Hq, a.Hkv, a.Lq, a.L, !ranges && !(a.softcap > 0.0f), ranges);
  if (a.mode >= 0) {   // a debug call says which
    plan.mode = static_cast<Mode>(a.mode);
    set_parts(plan, a.parts);
    if (plan.slots > 0 && (plan.mode > kRows32 || !ranges || !shares_out(a.B, a.Lq) || plan.slots < a.B)) return -2;
    plan.n_groups = static_cast<int>((static_cast<long long>(a.Hq / a.Hkv) * a.Lq + kModeRows[a.mode] - 1) / kModeRows[a.mode]);
  }
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  const size_t kv_bytes = decoded_bytes(plan, a.B, a.Hkv, a.L);
  if (kv_bytes > 0) {
    const Kv8Args d{ws, ws + kv_bytes, nullptr, nullptr, 0, a.L, a.B, a.Hkv, a.L, kD, 2, const_cast<void*>(a.k8),
                    const_cast<void*>(a.v8), const_cast<uint8_t*>(a.k_exp), const_cast<uint8_t*>(a.v_exp)};
    const int rd = launch_kv8_decode(d, stream);
    if (rd != 0) return rd;
  }
  if (plan.mode == kReadBack) {
    AttnArgs w{a.q, ws, ws + kv_bytes, a.k_seedmask, a.v_seedmask, a.seed_idx, a.n_seeds, a.B, a.Hq, a.Hkv, a.L, kD, a.out,
               a.lse, a.Lq, a.q0};
    const int rc = try_launch_attn_window_gqa(w, status, stream, false);
    return rc != kWindowGqaNotTaken ? rc : launch_attn_bf16_sm103(w, status, stream);
  }
  const long long grid = static_cast<long long>(plan.n_groups) * a.Hkv * (plan.slots > 0 ? plan.slots + a.B : a.B * static_cast<long long>(plan.nsplit));
  if (grid > 0x7fffffffLL) return -2;
  static ContextCache<int> setup;
  int unused = 0;
  const int rc = setup.get(&unused, [&](int&) {
    const auto limit = [](auto fn, size_t smem) {
      return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess;
    };
    // the register split inside the tile kernel assumes exactly kLaunchRegs per thread at launch; any other
    // count could leave setmaxnreg.inc waiting, so refuse to launch
    const auto registers = [](auto fn) {
      cudaFuncAttributes fa;
      return cudaFuncGetAttributes(&fa, fn) == cudaSuccess && fa.numRegs == kLaunchRegs;
    };
    for (int c = 0; c < 2; ++c) {
      for (int m = 0; m < 2; ++m)
        if (!limit(kRowsKernels[m][c], kRowsSmemBytes[m])) return -3;
      if (!limit(kTileKernels[c], kSmemBytes) || !limit(kPairKernels[c], kPairSmemBytes)) return -3;
      if (!registers(kTileKernels[c])) return -2;
    }
    return 0;
  });
  if (rc != 0) return rc;
  const bool few = plan.mode == kRows16 || plan.mode == kRows32;
  const bool decoded = plan.mode == kDecodedPairs;
  CUtensorMap tq{}, tk{}, tv{};
  if (few ? !make_u8_map_4d(&tk, a.k8, kD, a.L, a.Hkv, a.B, kBN) || !make_u8_map_4d(&tv, a.v8, kD, a.L, a.Hkv, a.B, kBN)
          : !make_bf16_map_4d(&tq, a.q, kD, static_cast<uint64_t>(rows), 1, 1, kBM))
    return -3;
  if (decoded &&
      (!make_bf16_map_4d(&tk, ws, kD, a.L, a.Hkv, a.B, kBN) || !make_bf16_map_4d(&tv, ws + kv_bytes, kD, a.L, a.Hkv, a.B, kBN)))
    return -3;
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
  p.part_o = reinterpret_cast<float*>(ws + 2 * kv_bytes);
  const size_t parts = part_rows(plan, a.B, a.Hq, a.Lq);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + parts * kD);
  if (plan.slots > 0) p.shares = reinterpret_cast<int2*>(p.part_ml + parts);
  p.status = status;
  p.rows = rows;
  p.B = a.B;
  p.n_seeds = a.n_seeds;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.Lq = a.Lq;
  p.Lk = a.L;
  p.q0 = a.q0;
  p.n_groups = plan.n_groups;
  p.nsplit = plan.nsplit;
  p.slots = plan.slots;
  p.joined = plan.joined ? 1 : 0;
  p.scale_log2 = log2e / root;
  const bool cap = a.softcap > 0.0f;
  const float softcap = fminf(fmaxf(a.softcap, kMinCap), kMaxCap);
  p.cap_log2 = softcap * log2e;
  p.cap_in = cap ? 2.0f * log2e / (softcap * root) : 0.0f;
  p.cap_x = cap ? 1.0f / (softcap * root) : 0.0f;
  p.cap_ref = cap ? fixed_reference(p.cap_log2) : -INFINITY;
  if (p.cap_ref != -INFINITY) {
    fixed_bytes(p.cap_log2, p.cap_ref, a.L, &p.v_lo, &p.v_hi);
    p.v_lo *= 0x01010101u, p.v_hi *= 0x01010101u;
  }
  const float tanh_poly[4] = {kTanh0, kTanh1, kTanh2, kTanh3};
  float power = p.cap_log2 * p.cap_x;
  for (int i = 0; i < 4; ++i, power *= p.cap_x * p.cap_x) p.cap_poly[i] = p.cap_ref != -INFINITY ? tanh_poly[i] * power : 0.0f;
  cudaLaunchAttribute pdl[1], attr[2];
  const int m = plan.mode == kRows16 ? 0 : 1;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(few ? kRowsThreads : kThreads),
                                      few ? kRowsSmemBytes[m] : decoded ? kPairSmemBytes : kSmemBytes, stream, pdl);
  attr[0] = pdl[0];
  if (plan.joined) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(plan.nsplit);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
  cudaError_t e;
  if (few) e = cudaLaunchKernelEx(&cfg, kRowsKernels[m][cap ? 1 : 0], tk, tv, p);
  else if (decoded) e = cudaLaunchKernelEx(&cfg, kPairKernels[cap ? 1 : 0], tq, tk, tv, p);
  else e = cudaLaunchKernelEx(&cfg, kTileKernels[cap ? 1 : 0], tq, p);
  if (e == cudaSuccess && parts > 0) {
    cfg = pdl_config(dim3(static_cast<unsigned>((rows + kCombineWarps - 1) / kCombineWarps)), dim3(kCombineWarps * 32), 0,
                     stream, pdl);
    e = cudaLaunchKernelEx(&cfg, attn_prefix8_combine_kernel, static_cast<const float*>(p.part_o),
                           static_cast<const float2*>(p.part_ml), plan.nsplit,
                           static_cast<const int2*>(p.shares), static_cast<long long>(a.Hq) * a.Lq, rows, p.out, p.lse);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
