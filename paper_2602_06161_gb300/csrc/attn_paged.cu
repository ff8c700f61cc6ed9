// attn_paged.cu - two-view window attention over a key/value memory in pages.
//
// k_pages, v_pages [n_pages, Hkv, page, 128] bf16; position t of sequence b is row t % page of the page table[b, t / page]. Query
// row r of head hq of sequence b sees the keys j of its sequence with key_lo <= j < key_hi, j < lens[b] and a page in the pool:
//   s_j = q . k_j / sqrt(d), capped: s_j = c tanh(s_j / c);  o = sum_j softmax(s)_j v_j,  lse = ln sum_j e^{s_j}
// A seed row's own column (its position is q0[b] + r), where it is among them, is the masked-input pair (k_i, v_i) instead. A row
// that sees no key gives o = 0, lse = -inf.
//
// The G = Hq / Hkv query heads of a KV head are packed: row p = g Lq + r of KV head (b, hkv) is query row r of head
// hkv G + g, and the packed rows are one run of the [B Hq Lq, D] view. Two ways, chosen by plan_of:
//   rows (16 or 32 a group)  few rows: bound by reading the memory
//   pairs (2 x 128 rows)     many rows: bound by the tensor cores and the softmax
// A KV tile is 128 keys, fetched a page (or half a page of 256) at a time, a copy each: the pool is one tensor of groups of eight rows, and a
// group is in shared memory its first 64 columns and then its last 64 (2 x 8 x 128 bytes, swizzled), so that pages of any size
// make the same tile, groups 2048 bytes apart. (A copy for each half of a page's columns, tiles of two halves: 64
// sequences of up to 8191 keys in pages of 16 took 231 us, in pages of 32 and more 197.) A position without a page is fetched from outside
// the tensor, which reads as zeros, and its scores count as unseen.
//
// What no row sees must not reach the sums: scores are taken out by selection, but a weight of zero times a value that is not finite
// is NaN. KV tiles of which some row does not see some key (the last one of a sequence, diagonals, windows, seeds' own
// columns) are looked through: a V row with an element that is not finite is set to zeros and reported, and the outputs of the rows that see
// it are made NaN instead. Tiles that all rows see whole are not (there the products give what they give). Sums and lse, which are of Q and K
// alone, stay what they are.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "attn_common.cuh"
#include "cluster.cuh"
#include "context.cuh"
#include "kernels.cuh"
#include "paged_ring.cuh"
#include "ptx.cuh"
#include "route.cuh"
#include "tmap.cuh"

namespace cover {
namespace {

constexpr int kD = 128;
constexpr int kBM = 128;                   // rows per Q tile (pairs)
constexpr int kBN = 128;                   // keys per KV tile
constexpr int kTileBytes = kBN * kD * 2;   // 32 KB
constexpr int kBoxBytes = kTileBytes / 2;  // of Q: 64 columns, 128-byte swizzled
constexpr int kGroupBytes = 2048, kGroupHalf = 1024;   // of K and V: eight rows, their first 64 columns
constexpr int kHalf = kBN / 2;
constexpr int kMaxTilePages = kBN / 16;
constexpr float kRescaleThreshold = 8.0f;  // log2 units
// Capped scores lie in [-C, C], C = cap log2(e). Up to C = kFixedCap (caps up to 55) the pairs kernel takes the same reference
// for every row, C - kFixedRange or 0, and looks for no maxima: weights lie in [2^(kFixedRange - 2 C), 2^kFixedRange], at least 2^-100, and sums
// over L keys hold values up to 2^66 / L.
constexpr float kFixedCap = 80.0f, kFixedRange = 60.0f;
constexpr int kSms = 152;                  // of this GPU
constexpr float kNan = __builtin_nanf("");

struct Params {
  const __nv_bfloat16* q;
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
  float* part_o;     // rows: [2 CTAs][kN][128]; pairs: [nsplit][rows][128]
  float2* part_ml;   // as part_o's rows: reference (log2 units) and sum
  int4* joins;       // rows: [CTAs] what the second kernel adds up
  int* status;
  long long rows;    // B * Hq * Lq
  int n_pages, M, page_log2, B, n_seeds, Hq, Hkv, G, Lq, n_groups, nsplit;
  int joined;        // CTAs of a cluster that share a unit's keys and add their results up themselves, or 0
  float scale_log2;  // log2(e) / sqrt(d)
  float cap_log2;    // cap * log2(e)
  float cap_in;      // 2 log2(e) / (cap sqrt(d))
  float cap_poly[4]; // coefficients of the capped score's polynomial, in powers of 1 / (cap sqrt(d))
  float cap_near;    // products up to this one may take it (below 0: none)
  float cap_ref;     // reference of all rows under a small cap (below 0: rows have their own)
};

// Keys of sequence b.
__device__ __forceinline__ int length_of(const Params& p, int b) {
  const long long most = static_cast<long long>(p.M) << p.page_log2;
  return static_cast<int>(min(static_cast<long long>(max(__ldg(p.lens + b), 0)), most));
}
// The keys lo .. hi - 1 that row i of [B Lq] sees of its sequence's len, held to 0 .. len; (0, 0) where it sees none.
__device__ __forceinline__ int2 keys_of(const Params& p, long long i, int len) {
  const int lo = p.key_lo != nullptr ? max(__ldg(p.key_lo + i), 0) : 0, hi = p.key_hi != nullptr ? min(__ldg(p.key_hi + i), len) : len;
  return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
}
// Entry of the table for the page that holds key `key` of sequence b, -1 where there is none.
__device__ __forceinline__ int page_of(const Params& p, int b, int key) {
  const int i = key >> p.page_log2;
  const int e = i < p.M ? __ldg(p.table + static_cast<size_t>(b) * p.M + i) : -1;
  return e >= 0 && e < p.n_pages ? e : -1;
}
// Position of query row r of a sequence whose first is at q0, or -1 where it is none that a key can have.
__device__ __forceinline__ int position_of(int q0, int r) {
  const long long at = static_cast<long long>(q0) + r;
  return at >= 0 && at <= 0x7fffffffLL ? static_cast<int>(at) : -1;
}

// Issues the copies of one KV tile whose first key is key0 into `tile`, a lane a page; entry: of the lane's page, -1 for none.
__device__ __forceinline__ void copy_tile(const CUtensorMap* tm, uint8_t* tile, uint64_t* full, int key0, int entry, int h, int Hkv,
                                          int page_log2, int lane) {
  const int rows_log2 = min(page_log2, 7);
  if (lane < kBN >> rows_log2) {
    const int within = page_log2 > 7 ? (key0 & ((1 << page_log2) - 1)) >> 3 : 0;
    const int group = entry < 0 ? -16 : ((entry * Hkv + h) << (page_log2 - 3)) + within;
    tma_load_4d(tile + (lane << rows_log2) * (kD * 2), tm, full, 0, 0, 0, group);
  }
}

// Whether V row `key` of a tile holds an element that is not finite; it is set to zeros then. One thread a key.
__device__ __forceinline__ bool screen_row(uint32_t tile, int key) {
  const uint32_t row = tile + (key >> 3) * kGroupBytes + (key & 7) * 128;
  uint32_t hit = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint4 c = lds128(row + (i >> 3) * kGroupHalf + (((i & 7) ^ (key & 7)) << 4));
    // an exponent of all ones carries into the sign's place
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) hit |= (w[e] & 0x7fff7fffu) + 0x00800080u;
  }
  const bool bad = (hit & 0x80008000u) != 0;
  if (bad) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i) sts128(row + (i >> 3) * kGroupHalf + ((i & 7) << 4), 0, 0, 0, 0);
  }
  return bad;
}

// The same for eight keys, by a warp: 2 KB in order, of which lane l reads 16 bytes of keys l / 8 and 4 + l / 8, of either half. Writes a byte
// of what was found.
__device__ __forceinline__ void screen_group(uint32_t group, uint8_t* found, int lane) {
  uint32_t hit[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 c = lds128(group + 512 * i + 16 * lane);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) hit[i & 1] |= (w[e] & 0x7fff7fffu) + 0x00800080u;
  }
  uint32_t bad = 0;
  if (__any_sync(0xffffffffu, ((hit[0] | hit[1]) & 0x80008000u) != 0)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lanes = __ballot_sync(0xffffffffu, (hit[h] & 0x80008000u) != 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) bad |= ((lanes >> (8 * k)) & 0xffu) != 0 ? 1u << (4 * h + k) : 0u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((bad >> (4 * (i & 1) + (lane >> 3))) & 1u) sts128(group + 512 * i + 16 * lane, 0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (lane == 0) *found = static_cast<uint8_t>(bad);
}

// Four columns of tensor memory.
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait4(uint32_t (&r)[4]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3])::"memory");
}

// Whether any of 128 or 256 threads of a named barrier says so.
template <int kAll>
__device__ __forceinline__ bool any_of(int barrier, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(x ? 1u : 0u), "r"(barrier), "n"(kAll)
      : "memory");
  return r != 0;
}
template <int kAll>
__device__ __forceinline__ void sync_of(int barrier) {
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(kAll) : "memory");
}

// Parts that a cluster's CTAs add up themselves: each stages its rows' accumulators [row][128] fp32 and (m, l) in its own
// shared memory, and CTA `rank` finishes the rows rank, rank + parts, .., a warp a row, reading all CTAs'. Rows' 16-byte
// pieces are swizzled, for threads that write a row each. A seed row's own pair is one part more, where the rows' slots are given: its score
// is in CTA 0's shared memory.
constexpr int kMaxJoined = 8;   // a cluster's portable size
__device__ __forceinline__ uint32_t staged_at(int row, int c4) { return row * (kD * 4) + ((c4 ^ (row & 31)) << 4); }

template <int kWarps>
__device__ __forceinline__ void join_rows(const Params& p, uint32_t staged, uint32_t ml, int n_rows, long long orow0, int rank, int parts,
                                          const int* slots = nullptr, uint32_t scores = 0, const __nv_bfloat16* values = nullptr) {
  const int lane = threadIdx.x & 31;
  for (int row = rank + parts * static_cast<int>(threadIdx.x >> 5); row < n_rows; row += parts * kWarps) {
    float2 mine = make_float2(-INFINITY, 0.0f);
    const int slot = slots != nullptr ? slots[row] : kNoSlot;
    float4 own = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (slot != kNoSlot) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(values + static_cast<size_t>(slot) * kD) + lane);
      own = make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                        __uint_as_float(v.y & 0xffff0000u));
      if (lane == kMaxJoined) {
        const uint32_t at = cluster_map(scores + 4 * row, 0);
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(mine.x) : "r"(at) : "memory");
        mine.y = mine.x == -INFINITY ? 0.0f : 1.0f;
      }
    }
    if (lane < parts) {
      const uint32_t at = cluster_map(ml + 8 * row, lane);
      asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(mine.x), "=f"(mine.y) : "r"(at) : "memory");
    }
    float4 x[kMaxJoined];
#pragma unroll
    for (int k = 0; k < kMaxJoined; ++k) {
      x[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (k < parts) {
        const uint32_t at = cluster_map(staged + staged_at(row, lane), k);
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[k].x), "=f"(x[k].y), "=f"(x[k].z), "=f"(x[k].w)
                     : "r"(at)
                     : "memory");
      }
    }
    float m = mine.x;   // (lanes up to kMaxJoined hold one)
#pragma unroll
    for (int d = kMaxJoined; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    m = __shfl_sync(0xffffffffu, m, 0);
    const float w = mine.x == -INFINITY ? 0.0f : ex2_approx(mine.x - m);
    float l = mine.x == -INFINITY ? mine.y : w * mine.y;   // (a sum of NaN is taken along)
#pragma unroll
    for (int d = kMaxJoined; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    l = __shfl_sync(0xffffffffu, l, 0);
    // (every part counts, those of weight zero too: a value that is not finite makes its column NaN there)
    const float w_own = __shfl_sync(0xffffffffu, w, kMaxJoined);
    float4 acc = make_float4(w_own * own.x, w_own * own.y, w_own * own.z, w_own * own.w);
#pragma unroll
    for (int k = 0; k < kMaxJoined; ++k) {
      const float wk = __shfl_sync(0xffffffffu, w, k);
      acc.x = fmaf(wk, x[k].x, acc.x), acc.y = fmaf(wk, x[k].y, acc.y), acc.z = fmaf(wk, x[k].z, acc.z), acc.w = fmaf(wk, x[k].w, acc.w);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    reinterpret_cast<uint2*>(p.out + (orow0 + row) * kD)[lane] =
        make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (lane == 0 && p.lse != nullptr) p.lse[orow0 + row] = (m + lg2_approx(l)) * 0.6931471805599453f;
  }
}
// The cluster's barriers around it, for warps that have no part in it.
__device__ __forceinline__ void join_pass() {
  __syncwarp();
  cluster_sync();
  cluster_sync();
}

// ---------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------
// The products are turned over, S^T = K Q^T (128 keys x kN rows), O^T += V^T P^T (128 columns x kN rows): a Q tile of 128 rows
// would cost the tensor cores and the softmax the same for one row as for 128. A softmax thread is a key. The rows' largest
// scores are only looked for when some score is above its row's reference by more than the threshold (one vote a tile); sums stay with
// the threads until the keys of a unit are through. Two streams take alternate KV tiles, with sums and an accumulator of their own; where
// units are of one tile, a stream takes a unit (256 sequences of 100 keys, 32 / 8 heads: 64 us by one stream after the other, 48 so).
//
// One CTA an SM, and the KV tiles of all units (sequence, KV head, group of rows) are one row of tiles of which every CTA takes an even
// share, whatever the lengths: a batch of sequences of 1 to 1000 tiles keeps all SMs reading until the end. Where a
// share's border cuts a unit, its CTAs leave their parts to a second kernel: at most two a CTA. Loads run on across units, so that a
// unit's end is hidden behind the next one's tiles.
// Few short sequences are done faster by a cluster a unit, whose CTAs share its tiles and add their results up through each other's
// shared memory: no look at the other sequences' lengths, no second kernel.
//
// Roles (512 threads): warps 0-3, 4-7 softmax of the streams; 8-11 look V tiles through; 12 products; 13 copies; 14 lays out what
// is to be done, tile by tile: pages, masks and rows, up to 8 tiles ahead.
// Shared memory: five tiles of K or V in the order K0 K1 V0 K2 V1 .. (paged_ring.cuh), Q of two units, P^T of two streams (rows of 128 bytes).
// With 32 rows a thread's 32 scores and 32 sums do not fit into its 128 registers beside the rest: 104 to 216 bytes are spilled.
// Tensor memory: S0 | S1 | O0 | O1, kN columns each.
constexpr int kRowsThreads = 512;
constexpr int kScreenWarp = 8, kRowsMmaWarp = 12, kRowsCopyWarp = 13, kRowsPlanWarp = 14;
constexpr int kSlots = paged_ring::kSlots, kRing = 8, kUnits = 8;

struct TileJob {
  int page[kMaxTilePages];   // entries of its pages, -1 for none
  int key0, h, q_row;
  uint32_t valid;            // bit i: page i is there
  int first, last;           // of the unit's tiles in this CTA
  int partial;               // some row does not see some key
  int unit;                  // number of the unit in this CTA
};

template <int kN>
constexpr int kQueries = 2;   // units whose Q is in shared memory

template <int kN>
struct RowsSmem {
  uint8_t kv[kSlots][kTileBytes];
  uint8_t q[kQueries<kN>][kN * kD * 2];
  uint8_t pt[2][kBN * 128];
  uint64_t k_full[paged_ring::kBarriers], v_full[paged_ring::kBarriers], empty[kSlots];
  uint64_t q_full[kQueries<kN>], q_empty[kQueries<kN>];
  uint64_t job_full[kRing], job_empty[kRing], v_clean[kRing];
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  uint64_t s_full[2], p_full[2], o_full[2], drain;
  TileJob job[kRing];
  uint4 nan_keys[kRing];
  int4 row[kUnits][kN];      // per unit: keys lo, hi, position of a seed row or -1, its slot
  int4 unit[kUnits];         // tiles here, rows, first row of [B Hq Lq], part's place: -1 whole, -2 joined, else its number
  int2 unit_mask[kUnits];    // masked-input rows of the KV head, whether the unit's first tile is here
  float4 fin[2][kN];         // weights of the two accumulators and of the masked-input value, 1 / l
  float m[2][kN], step[2][kN], factor[2][kN];
  int unseen[2][kN], any_unseen[2];
  int bad[2][kN];            // whether the row sees a V row that was set to zeros
  float red[2][4][kN];
  float s_self[2][kN];
  int slot[kN];
  float2 ml[kN];             // joined in a cluster: the rows' references and sums
  long long scan[kRowsThreads / 32];
  long long t0, t1, before;  // this CTA's tiles, those before the first sequence of them
  int b0;
  uint32_t tmem_base;
  int abort;
};

// First of the tiles of CTA c of n, of T.
__device__ __forceinline__ long long share_start(long long c, long long n, long long T) { return c * T / n; }

// KV tiles of a unit of sequence b, and the first of them; one at least. One warp, or (kAlone) one thread.
template <bool kAlone>
__device__ __forceinline__ int2 tiles_of(const Params& p, int b) {
  const int len = length_of(p, b);
  int lo = 0x7fffffff, hi = 0;
  if (p.key_lo == nullptr && p.key_hi == nullptr) {
    lo = 0, hi = len;
  } else {
    for (int r = kAlone ? 0 : threadIdx.x & 31; r < p.Lq; r += kAlone ? 1 : 32) {
      const int2 k = keys_of(p, static_cast<long long>(b) * p.Lq + r, len);
      if (k.y > 0) lo = min(lo, k.x), hi = max(hi, k.y);
    }
    if (!kAlone) lo = __reduce_min_sync(0xffffffffu, lo), hi = __reduce_max_sync(0xffffffffu, hi);
  }
  if (hi == 0) return make_int2(1, 0);
  const int first = lo / kBN;
  return make_int2((hi - 1) / kBN + 1 - first, first);
}

template <int kN, bool kCap, bool kJoined>
__global__ void __launch_bounds__(kRowsThreads, 1)
    attn_paged_rows_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                           const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  using Sm = RowsSmem<kN>;
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr uint32_t kTmem = 4 * kN;
  constexpr int kQ = kQueries<kN>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (warp == kRowsMmaWarp) {
    if (lane == 0) {
      for (int i = 0; i < kSlots; ++i) mbar_init(&sm.empty[i], 1);
      for (int i = 0; i < paged_ring::kBarriers; ++i) mbar_init(&sm.k_full[i], 1), mbar_init(&sm.v_full[i], 1);
      for (int i = 0; i < kRing; ++i) {
        mbar_init(&sm.job_full[i], 1);
        mbar_init(&sm.job_empty[i], 10);   // copies, products, four warps that look V through, four of a stream
        mbar_init(&sm.v_clean[i], 128);
      }
      for (int i = 0; i < kQ; ++i) mbar_init(&sm.q_full[i], 1), mbar_init(&sm.q_empty[i], 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], 128);
      }
      for (int i = 0; i < kUnits; ++i) mbar_init(&sm.unit_full[i], 1), mbar_init(&sm.unit_empty[i], 8);
      mbar_init(&sm.o_full[0], 1), mbar_init(&sm.o_full[1], 1);
      mbar_init(&sm.drain, 1);
      sm.abort = 0;
      sm.b0 = 0;
      fence_mbar_init();
      tma_prefetch_desc(&tm_q);
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
    }
    __syncwarp();
    tmem_alloc(&sm.tmem_base, kTmem);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = sm.tmem_base;
  griddep_wait();
  griddep_launch_dependents();

  // ---------------- the CTA's share of all tiles ----------------
  const int n_packed = p.G * p.Lq;
  const int heads = p.Hkv * p.n_groups;   // units of a sequence (at most B Hq Lq)
  long long t0, t1, all = 0, n_ctas = 0, c = blockIdx.x;
  int b0;
  long long before0 = 0;   // tiles before sequence b0's
  int tile0 = 0;           // joined: the CTA's first tile of the sequence's
  if (kJoined) {
    // tiles counted from the sequence's first: a part of those of the cluster's unit
    const int u = static_cast<int>(blockIdx.x) / p.joined, rank = static_cast<int>(blockIdx.x) % p.joined;
    b0 = u / heads;
    int line = 0;
    if (warp == kRowsCopyWarp && lane * 32 < p.M)   // the table's first lines are on their way to L1 while the length is
      asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(line) : "l"(p.table + static_cast<size_t>(b0) * p.M + lane * 32));
    const int2 tiles = tiles_of<false>(p, b0);
    asm volatile("" ::"r"(line));
    const int share = tiles.x / p.joined, more = tiles.x % p.joined, j = rank * share + min(rank, more);
    t0 = static_cast<long long>(u % heads) * tiles.x + j;
    t1 = t0 + share + (rank < more ? 1 : 0);
    tile0 = tiles.y + j;
  } else {
    const int each = (p.B + kRowsThreads - 1) / kRowsThreads;           // sequences of a thread
    const int b_lo = min(tid * each, p.B), b_hi = min(b_lo + each, p.B);
    long long mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += static_cast<long long>(tiles_of<true>(p, b).x) * heads;
    long long incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += x;
    }
    if (lane == 31) sm.scan[warp] = incl;
    __syncthreads();
    long long before = 0;
    for (int w = 0; w < kRowsThreads / 32; ++w) {
      if (w < warp) before += sm.scan[w];
      all += sm.scan[w];
    }
    n_ctas = min(static_cast<long long>(gridDim.x), all);
    t0 = c < n_ctas ? share_start(c, n_ctas, all) : 0, t1 = c < n_ctas ? share_start(c + 1, n_ctas, all) : 0;
    before += incl - mine;
    if (t0 < t1 && t0 >= before && t0 < before + mine) {
      int b = b_lo;
      for (long long x; before + (x = static_cast<long long>(tiles_of<true>(p, b).x) * heads) <= t0; ++b) before += x;
      sm.b0 = b;
      sm.before = before;
    }
    __syncthreads();
    b0 = sm.b0;
    before0 = sm.before;
  }
  const int n = static_cast<int>(t1 - t0);   // tiles of this CTA

  if (warp == kRowsPlanWarp) {
    // ---------------- what is to be done ----------------
    bool ok = true;
    int b = b0, g = 0, unit = 0;
    long long first = before0;   // of the sequence's tiles
    int2 tiles = n > 0 ? tiles_of<false>(p, b) : make_int2(1, 0);
    if (!kJoined && n == 0 && lane == 0) p.joins[blockIdx.x] = make_int4(0, 0, 0, 0);
    bool joined = false;
    for (long long t = t0; t < t1 && ok; ++unit) {
      for (long long all_of; t >= first + (all_of = static_cast<long long>(tiles.x) * heads); ) first += all_of, tiles = tiles_of<false>(p, ++b);
      int u, j;
      if (t - first <= 0x7fffffffLL) u = static_cast<int>(t - first) / tiles.x, j = static_cast<int>(t - first) % tiles.x;
      else u = static_cast<int>((t - first) / tiles.x), j = static_cast<int>((t - first) % tiles.x);
      const int nt = static_cast<int>(min(static_cast<long long>(tiles.x - j), t1 - t));
      const int h = u / p.n_groups, p0 = (u % p.n_groups) * kN, n_rows = min(kN, n_packed - p0);
      const long long rowbase = (static_cast<long long>(b) * p.Hq + h * p.G) * p.Lq;
      const int len = length_of(p, b), buf = unit % kUnits;
      const int pages = kBN >> min(p.page_log2, 7);
      // (loads that depend on nothing else first)
      int first_pos = 0, first_seed = 0;
      if (p.n_seeds > 0) {
        first_pos = __ldg(p.q0 + b);
        if (lane < p.n_seeds) first_seed = __ldg(p.seed_idx + static_cast<size_t>(b) * p.n_seeds + lane);
      }
      int entry = lane < pages ? page_of(p, b, (tiles.y + j) * kBN + (lane << min(p.page_log2, 7))) : -1;
      if (unit >= kUnits) ok = warp_wait(&sm.unit_empty[buf], (unit / kUnits - 1) & 1, &sm.abort);
      if (!ok) break;
      // seed rows: the rows stand at up to kN positions, r itself or r - r0 around Lq
      const int r0 = p.Lq <= kN ? 0 : p0 % p.Lq;
      if (p.n_seeds > 0) {
        if (lane < kN) sm.slot[lane] = kNoSlot;
        __syncwarp();
        for (int s = lane; s < p.n_seeds; s += 32) {
          const int seed = s == lane ? first_seed : __ldg(p.seed_idx + static_cast<size_t>(b) * p.n_seeds + s);
          const long long at = static_cast<long long>(seed) - first_pos;
          if (at < 0 || at >= p.Lq) continue;
          const int i = static_cast<int>(at >= r0 ? at - r0 : at - r0 + p.Lq);
          if (i < kN) atomicMin(&sm.slot[i], s);
        }
        __syncwarp();
      }
      int all_lo = 0, all_hi = 0x7fffffff, own_lo = 0x7fffffff, own_hi = -1;   // keys that every row sees, seed rows' positions
      if (lane < kN) {
        int4 row = make_int4(0, 0, -1, 0);
        if (lane < n_rows) {
          const int r = (p0 + lane) % p.Lq;
          const int2 k = keys_of(p, static_cast<long long>(b) * p.Lq + r, len);
          row.x = k.x, row.y = k.y;
          if (p.n_seeds > 0) {
            const int slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq], at = position_of(first_pos, r);
            if (slot != kNoSlot && at >= k.x && at < k.y && page_of(p, b, at) >= 0) {
              row.z = at, row.w = slot;
              own_lo = own_hi = at;
            }
          }
          all_lo = row.x, all_hi = row.y;   // (a row that sees nothing makes every tile partial)
        }
        sm.row[buf][lane] = row;
      }
      all_lo = __reduce_max_sync(0xffffffffu, all_lo), all_hi = __reduce_min_sync(0xffffffffu, all_hi);
      own_lo = __reduce_min_sync(0xffffffffu, own_lo), own_hi = __reduce_max_sync(0xffffffffu, own_hi);
      const bool whole = nt == tiles.x;
      __syncwarp();
      if (lane == 0) {
        // a part that begins its unit comes last in its CTA, any other first
        const int place = kJoined ? -2 : whole ? -1 : static_cast<int>(2 * c) + (j == 0 ? 1 : 0);
        sm.unit[buf] = make_int4(nt, n_rows, static_cast<int>(rowbase + p0), place);
        sm.unit_mask[buf] = make_int2(static_cast<int>((static_cast<long long>(b) * p.Hkv + h)), j == 0 ? 1 : 0);
        if (j == 0 && !whole && !kJoined) {
          // the unit's last tile is of CTA ((tile + 1) n - 1) / T
          const long long last = first + static_cast<long long>(u + 1) * tiles.x - 1;
          p.joins[blockIdx.x] = make_int4(static_cast<int>(((last + 1) * n_ctas - 1) / all - c) + 1, n_rows, static_cast<int>(rowbase + p0), 0);
          joined = true;
        }
        mbar_arrive(&sm.unit_full[buf]);
      }
      for (int i = 0; i < nt && ok; ++i, ++g) {
        const int key0 = (tiles.y + j + i) * kBN, at = g % kRing;
        if (i > 0) entry = lane < pages ? page_of(p, b, key0 + (lane << min(p.page_log2, 7))) : -1;
        if (g >= kRing) ok = warp_wait(&sm.job_empty[at], (g / kRing - 1) & 1, &sm.abort);
        if (!ok) break;
        TileJob& job = sm.job[at];
        const uint32_t valid = __ballot_sync(0xffffffffu, entry >= 0);
        if (lane < pages) job.page[lane] = entry;
        if (lane == 0) {
          job.key0 = key0;
          job.h = h;
          job.q_row = static_cast<int>(rowbase + p0);
          job.valid = valid;
          job.first = i == 0;
          job.last = i == nt - 1;
          job.partial = key0 < all_lo || all_hi - key0 < kBN || valid != (1u << pages) - 1u || (own_hi >= key0 && own_lo - key0 < kBN);
          job.unit = unit;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.job_full[at]);
      }
      t += nt;
    }
    if (lane == 0 && n > 0 && !joined && !kJoined) p.joins[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 80);
      sm.abort = 1;
    }
  } else if (warp == kRowsCopyWarp) {
    // ---------------- copies ----------------
    bool ok = true;
    int issued = 0, q_issued = 0;   // tiles of K and V, units
    const int rows_log2 = min(p.page_log2, 7);
    const auto lookup = [&](int tile) { return lane < kBN >> rows_log2 ? page_of(p, b0, tile * kBN + (lane << rows_log2)) : -1; };
    // joined: the pages of the CTA's tiles, looked up here and a tile ahead (a job from the planning warp takes a microsecond more)
    int entry_v = -1, entry_k = -1, entry_next = kJoined && n > 0 ? lookup(tile0) : -1;
    const int u0 = kJoined ? static_cast<int>(blockIdx.x) / p.joined % heads : 0;
    for (int i = 0; i < 2 * n && ok; ++i) {
      const paged_ring::Copy copy = paged_ring::copy_at(i, n);
      const bool is_v = copy.is_v;
      const int g = copy.tile, at = g % kRing, slot = paged_ring::slot_of(i);
      uint64_t* const full = (is_v ? sm.v_full : sm.k_full) + paged_ring::barrier_of(g);
      if (is_v == kJoined) ok = warp_wait(&sm.job_full[at], (g / kRing) & 1, &sm.abort);   // (joined: for the arrival below alone)
      if (ok && i >= kSlots) ok = warp_wait(&sm.empty[slot], (i / kSlots - 1) & 1, &sm.abort);
      if (!ok) break;
      int entry, key0, h;
      if (kJoined) {
        if (!is_v) {
          entry_v = entry_k;
          entry_k = entry_next;
          if (g + 1 < n) entry_next = lookup(tile0 + g + 1);
        }
        entry = is_v && i < 2 * n - 1 ? entry_v : entry_k;
        key0 = (tile0 + g) * kBN;
        h = u0 / p.n_groups;
      } else {
        const TileJob& job = sm.job[at];
        entry = job.page[lane % kMaxTilePages], key0 = job.key0, h = job.h;
      }
      if (!is_v && (kJoined ? i == 0 : sm.job[at].first != 0)) {
        const int unit = kJoined ? 0 : sm.job[at].unit, buf = unit % kQ;
        const int q_row = kJoined ? static_cast<int>((static_cast<long long>(b0) * p.Hq + h * p.G) * p.Lq + (u0 % p.n_groups) * kN)
                                  : sm.job[at].q_row;
        if (unit >= kQ) ok = warp_wait(&sm.q_empty[buf], (unit / kQ - 1) & 1, &sm.abort);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&sm.q_full[buf], kN * kD * 2);
          for (int half = 0; half < 2; ++half) tma_load_4d(sm.q[buf] + half * kN * 128, &tm_q, &sm.q_full[buf], 64 * half, q_row, 0, 0);
        }
        q_issued = unit + 1;
      }
      if (lane == 0) mbar_arrive_expect_tx(full, kTileBytes);
      __syncwarp();
      copy_tile(is_v ? &tm_v : &tm_k, sm.kv[slot], full, key0, entry, h, p.Hkv, p.page_log2, lane);
      __syncwarp();
      if (is_v && lane == 0) mbar_arrive(&sm.job_empty[at]);
      issued = i + 1;
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 81);
      sm.abort = 1;
    }
    // every copy lands before the CTA's shared memory is released, whatever the other roles did
    if (lane == 0) {
      for (int f = max(0, issued - kSlots); f < issued; ++f) {
        const paged_ring::Copy copy = paged_ring::copy_at(f, n);
        mbar_wait((copy.is_v ? sm.v_full : sm.k_full) + paged_ring::barrier_of(copy.tile), paged_ring::phase_of(copy.tile) & 1, nullptr);
      }
      for (int f = max(0, q_issued - kQ); f < q_issued; ++f) mbar_wait(&sm.q_full[f % kQ], (f / kQ) & 1, nullptr);
    }
  } else if (warp == kRowsMmaWarp) {
    if (lane == 0 && n > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_s = idesc_bf16_f32(kBN, kN, false, false);
      constexpr uint32_t id_o = idesc_bf16_f32(kD, kN, true, true);
      // descriptors are added up in their lower words; K's and V's upper words are the same, and Q's and P's
      const uint64_t dk = sdesc_sw128(smem_u32(sm.kv[0]), 16, kGroupBytes), dv = sdesc_sw128(smem_u32(sm.kv[0]), kGroupHalf, kGroupBytes);
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[0]), 16, 1024), dp = sdesc_sw128(smem_u32(sm.pt[0]), 16, 1024);
      const uint32_t k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv), q_lo = static_cast<uint32_t>(dq),
                     p_lo = static_cast<uint32_t>(dp), kv_hi = static_cast<uint32_t>(dk >> 32), hi = static_cast<uint32_t>(dq >> 32);
      const auto desc = [](uint32_t lo, uint32_t up) { return (static_cast<uint64_t>(up) << 32) | lo; };
      const auto wait = [&](uint64_t* bar, int phase) {
        const bool done = mbar_wait(bar, phase & 1, &sm.abort);
        if (done) tc_fence_after_sync();
        return done;
      };
      bool ok = true;
      int unit = -1;   // of the last S
      // S^T[g & 1] = K(tile g) . Q^T
      const auto issue_s = [&](int g) {
        const int at = g % kRing, slot = paged_ring::slot_of(paged_ring::copy_of_k(g));
        ok = wait(&sm.job_full[at], g / kRing) && wait(&sm.k_full[paged_ring::barrier_of(g)], paged_ring::phase_of(g));
        if (!ok) return;
        if (sm.job[at].first) {
          ++unit;
          ok = wait(&sm.q_full[unit % kQ], unit / kQ);
          if (!ok) return;
        }
        const uint32_t k = k_lo + ((slot * kTileBytes) >> 4), q = q_lo + (((unit % kQ) * kN * kD * 2) >> 4);
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk)
          umma_ss(tbase + (g & 1) * kN, desc(k + (((kk >> 2) * kGroupHalf + (kk & 3) * 32) >> 4), kv_hi),
                  desc(q + (((kk >> 2) * kN * 128 + (kk & 3) * 32) >> 4), hi), id_s, kk > 0 ? 1u : 0u);
        umma_commit(&sm.s_full[g & 1]);
        umma_commit(&sm.empty[slot]);
        if (sm.job[at].last) umma_commit(&sm.q_empty[unit % kQ]);
      };
      for (int g = 0; g < 2 && g < n && ok; ++g) issue_s(g);
      int in_unit = 0;   // the tile's number in its unit
      for (int g = 0; g < n && ok; ++g, ++in_unit) {
        const int at = g % kRing, slot = paged_ring::slot_of(paged_ring::copy_of_v(g, n)), s = g & 1;
        ok = wait(&sm.v_full[paged_ring::barrier_of(g)], paged_ring::phase_of(g)) && wait(&sm.v_clean[at], g / kRing) && wait(&sm.p_full[s], g >> 1);
        if (!ok) break;
        if (sm.job[at].first) in_unit = 0;
        const bool last = sm.job[at].last != 0;
        const uint32_t v = v_lo + ((slot * kTileBytes) >> 4), pt = p_lo + ((s * kBN * 128) >> 4);
        // O^T[s] (+)= V(tile g)^T . P^T
#pragma unroll
        for (int kk = 0; kk < kBN / 16; ++kk)
          umma_ss(tbase + (2 + s) * kN, desc(v + ((kk * 2 * kGroupBytes) >> 4), kv_hi), desc(pt + ((kk * 2048) >> 4), hi), id_o,
                  (in_unit > 1 || kk > 0) ? 1u : 0u);
        umma_commit(&sm.empty[slot]);
        if (last && (in_unit > 0 || kJoined || s == 0)) umma_commit(&sm.o_full[0]);
        if (last && (in_unit > 0 || kJoined || s == 1)) umma_commit(&sm.o_full[1]);   // (a unit of one tile is its stream's alone)
        mbar_arrive(&sm.job_empty[at]);
        if (g + 2 < n) issue_s(g + 2);
      }
      if (!ok) {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 82);
        sm.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&sm.drain);
      mbar_wait(&sm.drain, 0, nullptr);
    }
    __syncwarp();
  } else if (warp >= kScreenWarp && warp < kRowsMmaWarp) {
    // ---------------- V rows that are not finite (thread = key) ----------------
    const int key = tid - kScreenWarp * 32;
    bool ok = true;
    for (int g = 0; g < n; ++g) {
      const int at = g % kRing, slot = paged_ring::slot_of(paged_ring::copy_of_v(g, n));
      ok = warp_wait(&sm.job_full[at], (g / kRing) & 1, &sm.abort) &&
           warp_wait(&sm.v_full[paged_ring::barrier_of(g)], paged_ring::phase_of(g) & 1, &sm.abort);
      if (!ok) break;
      uint32_t bad = 0;
      if (sm.job[at].partial) {
        bad = __ballot_sync(0xffffffffu, screen_row(smem_u32(sm.kv[slot]), key));
        fence_proxy_async_smem();
      }
      if (lane == 0) reinterpret_cast<uint32_t*>(&sm.nan_keys[at])[key >> 5] = bad;
      __syncwarp();
      mbar_arrive(&sm.v_clean[at]);
      if (lane == 0) mbar_arrive(&sm.job_empty[at]);
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 83);
      sm.abort = 1;
    }
  } else if (warp < kScreenWarp) {
    // ---------------- softmax (thread = key of a KV tile) ----------------
    const int stream = warp >> 2, key = tid & (kBN - 1), w4 = warp & 3;
    const uint32_t quad = tbase + (static_cast<uint32_t>(w4 * 32) << 16);
    const uint32_t s_addr = quad + stream * kN, o_addr = quad + (2 + stream) * kN;
    const float* m = sm.m[stream];
    const uint32_t pt = smem_u32(sm.pt[stream]) + key * 128;
    const uint32_t sw = static_cast<uint32_t>(key & 7) << 4;
    const int page_rows = min(p.page_log2, 7);
    const uint32_t staged = smem_u32(sm.kv[0]);   // joined: every copy and product is complete by then
    bool ok = true;
    int g = 0;
    if (n == 0) {   // joined: a part without keys
      if (tid < kN) sm.ml[tid] = make_float2(-INFINITY, 0.0f);
      if (kJoined)
        for (int i = tid; i < kN * kD / 4; i += 2 * kBN) sts128(staged + 16 * i, 0, 0, 0, 0);
    }
    for (int first_unit = 0, o_waits = 0; g < n;) {
      // Units of one tile, two in turn, are done by a stream each at the same time.
      ok = warp_wait(&sm.unit_full[first_unit % kUnits], (first_unit / kUnits) & 1, &sm.abort);
      const bool alone = ok && sm.unit[first_unit % kUnits].x == 1 && !kJoined;
      bool two = alone && g + 1 < n;
      if (two) {
        ok = warp_wait(&sm.unit_full[(first_unit + 1) % kUnits], ((first_unit + 1) / kUnits) & 1, &sm.abort);
        two = ok && sm.unit[(first_unit + 1) % kUnits].x == 1;
      }
      if (any_of<256>(1, !ok)) {
        ok = false;
        break;
      }
      const bool second = alone && (g & 1) != stream;   // the stream has the next unit, if that is one of a tile
      const bool idle = second && !two;
      const int unit = first_unit + (second && two ? 1 : 0), buf = unit % kUnits;
      const int4 info = sm.unit[buf];
      const int nt = alone ? (two ? 2 : 1) : info.x, n_rows = idle ? 0 : info.y;   // tiles of this turn
      const long long orow0 = info.z;
      const int place = info.w;
      const bool own_rows = sm.unit_mask[buf].y != 0 && p.n_seeds > 0;   // the masked-input pairs are added where the unit begins
      const size_t masked0 = static_cast<size_t>(sm.unit_mask[buf].x) * p.n_seeds;
      float* const s_self_of = sm.s_self[alone ? stream : 0];
      float4* const fin = sm.fin[alone ? stream : 0];
      const bool leads = alone || stream == 0;   // of the unit's streams
      const auto sync_unit = [&] {
        if (alone) sync_of<128>(2 + stream);
        else sync_of<256>(1);
      };
      if (key < kN) {
        sm.m[stream][key] = 0.0f;
        sm.unseen[stream][key] = key < n_rows ? 1 : 0;
        sm.bad[stream][key] = 0;
        if (key == 0) sm.any_unseen[stream] = 1;
        if (leads) s_self_of[key] = -INFINITY;
      }
      sync_unit();
      if (own_rows) {
        // the seed rows' own scores (log2 units): a warp a row, four columns a lane
        for (int i = alone ? w4 : warp; i < n_rows; i += alone ? 4 : 8) {
          const int4 row = sm.row[buf][i];
          if (row.z < 0) continue;
          const uint2 a = __ldg(reinterpret_cast<const uint2*>(p.q + (orow0 + i) * kD) + lane);
          const uint2 b = __ldg(reinterpret_cast<const uint2*>(p.k_seedmask + (masked0 + row.w) * kD) + lane);
          float dot = __uint_as_float(a.x << 16) * __uint_as_float(b.x << 16);
          dot = fmaf(__uint_as_float(a.x & 0xffff0000u), __uint_as_float(b.x & 0xffff0000u), dot);
          dot = fmaf(__uint_as_float(a.y << 16), __uint_as_float(b.y << 16), dot);
          dot = fmaf(__uint_as_float(a.y & 0xffff0000u), __uint_as_float(b.y & 0xffff0000u), dot);
          for (int d = 16; d >= 1; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
          if (lane == 0) s_self_of[i] = kCap ? capped(dot, p.cap_in, p.cap_log2) : dot * p.scale_log2;
        }
      }
      float l[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) l[i] = 0.0f;
      const int g0 = g;
      for (; g < g0 + nt; ++g) {
        if ((g & 1) != stream) continue;
        const int at = g % kRing;
        ok = warp_wait(&sm.job_full[at], (g / kRing) & 1, &sm.abort) && warp_wait(&sm.s_full[stream], (g >> 1) & 1, &sm.abort);
        const bool partial = ok && sm.job[at].partial != 0;
        float t[kN];        // scores less the references, in log2 units
        bool over = !ok;    // a warp whose wait gave up votes all the same: the stream's barriers take 128 threads
        if (ok) {
          tc_fence_after_sync();
#pragma unroll
          for (int c0 = 0; c0 < kN; c0 += 16) {
            uint32_t x[16];
            tmem_ld16(s_addr + c0, x);
            tmem_ld_wait16(x);
            float far = 0.0f;
            if (kCap) {
#pragma unroll
              for (int e = 0; e < 16; e += 2) far = fmax3(far, fabsf(__uint_as_float(x[e])), fabsf(__uint_as_float(x[e + 1])));
            }
            if (kCap && __any_sync(0xffffffffu, !(far <= p.cap_near))) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                if (e % 4 == 0 && c0 + e >= n_rows) break;   // (a cap is not worked out for rows that are none)
                t[c0 + e] = capped(__uint_as_float(x[e]), p.cap_in, p.cap_log2) - m[c0 + e];
              }
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float f = __uint_as_float(x[e]), z = f * f;
                // (the pairs kernel's polynomial of a cap)
                if (kCap) t[c0 + e] = fmaf(f, fmaf(z, fmaf(z, fmaf(z, p.cap_poly[3], p.cap_poly[2]), p.cap_poly[1]), p.cap_poly[0]), -m[c0 + e]);
                else t[c0 + e] = fmaf(f, p.scale_log2, -m[c0 + e]);
              }
            }
          }
          if (partial) {
            const int pos = sm.job[at].key0 + key;
            const bool held = ((sm.job[at].valid >> (key >> page_rows)) & 1u) != 0;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
              if (i >= n_rows) break;
              const int4 row = sm.row[buf][i];
              if (!held || pos < row.x || pos >= row.y || pos == row.z) t[i] = -INFINITY;
            }
          }
#pragma unroll
          for (int i = 0; i < kN; ++i) over |= i < n_rows && t[i] > kRescaleThreshold;
          over |= sm.any_unseen[stream] != 0;
          __syncwarp();
        }
        if (any_of<128>(2 + stream, over)) {
          if (any_of<128>(2 + stream, !ok)) {
            ok = false;
            break;
          }
          // new references: the rows' maxima where they are above the old ones by more than the threshold
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            if (i >= n_rows) break;   // (references of rows that are none are anything)
            const int top = __reduce_max_sync(0xffffffffu, ordered(t[i] == t[i] ? t[i] : -INFINITY));
            if (lane == (i & 31)) sm.red[stream][w4][i] = from_ordered(top);
          }
          sync_of<128>(2 + stream);
          if (key < kN) {
            const float up = fmaxf(fmaxf(sm.red[stream][0][key], sm.red[stream][1][key]),
                                   fmaxf(sm.red[stream][2][key], sm.red[stream][3][key]));
            // a row's first keys set its reference, wherever they lie
            const bool first = sm.unseen[stream][key] != 0 && up > -INFINITY;
            const float step = first || up > kRescaleThreshold ? up : 0.0f;
            sm.step[stream][key] = step;
            sm.factor[stream][key] = first ? 0.0f : ex2_approx(-step);
            sm.m[stream][key] = m[key] + step;
            if (first) sm.unseen[stream][key] = 0;
            const uint32_t mask = kN == 32 ? 0xffffffffu : 0xffffu;
            const uint32_t still = __ballot_sync(mask, sm.unseen[stream][key] != 0);
            if (key == 0) sm.any_unseen[stream] = still != 0 ? 1 : 0;
          }
          sync_of<128>(2 + stream);
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            t[i] -= sm.step[stream][i];
            l[i] *= sm.factor[stream][i];
          }
          if (g - g0 >= 2) {
            // O holds the stream's earlier products of the unit (complete: the commit of this S came after them)
#pragma unroll
            for (int c0 = 0; c0 < kN; c0 += 16) {
              uint32_t o[16];
              tmem_ld16(o_addr + c0, o);
              tmem_ld_wait16(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * sm.factor[stream][c0 + e]);
              tmem_st16(o_addr + c0, o);
            }
            tmem_st_wait();
          }
        }
#pragma unroll
        for (int c0 = 0; c0 < kN; c0 += 8) {
          if (c0 >= n_rows) break;   // (columns of P^T behind the rows hold anything: so do those of O^T)
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float e0 = ex2_approx(t[c0 + 2 * e]), e1 = ex2_approx(t[c0 + 2 * e + 1]);
            l[c0 + 2 * e] += e0;
            l[c0 + 2 * e + 1] += e1;
            w[e] = pack_bf16x2(e0, e1);   // V's operands are bf16, so P's have to be; a weight is off by 2^-8 of itself
          }
          sts128(pt + (static_cast<uint32_t>(c0 * 2) ^ sw), w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();
        mbar_arrive(&sm.p_full[stream]);
        if (partial) {
          // V has been looked through by now: the rows that see a row of it that is not finite are NaN
          ok = warp_wait(&sm.v_clean[at], (g / kRing) & 1, &sm.abort);
          if (ok && ((reinterpret_cast<const uint32_t*>(&sm.nan_keys[at])[key >> 5] >> (key & 31)) & 1u) != 0) {
            const int pos = sm.job[at].key0 + key;
            const bool held = ((sm.job[at].valid >> (key >> page_rows)) & 1u) != 0;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
              const int4 row = sm.row[buf][i];
              if (held && pos >= row.x && pos < row.y && pos != row.z) sm.bad[stream][i] = 1;
            }
          }
          __syncwarp();
          if (!ok && lane == 0) sm.abort = 1;   // (the next wait ends the loop, at a vote)
        }
        if (lane == 0) mbar_arrive(&sm.job_empty[at]);
      }
      if (ok && !idle) ok = warp_wait(&sm.o_full[stream], o_waits++ & 1, &sm.abort);
      if (alone ? any_of<128>(2 + stream, !ok) : any_of<256>(1, !ok)) ok = false;   // (of a unit's threads all or none go on)

      // ---------------- the rows' results ----------------
      if (ok) {
        tc_fence_after_sync();
        // sums over the warp: each step adds up and hands on half of the rows, until a lane has one. (The code of a unit's end is kept short: in
        // a call of a few tiles it runs once, out of a cold instruction cache. Unrolled over all rows it took 1.9 us.)
#pragma unroll
        for (int d = 16, left = kN; left > 1; d >>= 1, left >>= 1) {
          const bool upper = (lane & d) != 0;
#pragma unroll
          for (int i = 0; i < left / 2; ++i) {
            const float mine = upper ? l[i + left / 2] : l[i], other = upper ? l[i] : l[i + left / 2];
            l[i] = mine + __shfl_xor_sync(0xffffffffu, other, d);
          }
        }
        if (kN == 16) l[0] += __shfl_xor_sync(0xffffffffu, l[0], 1);
        sm.red[stream][w4][kN == 16 ? lane >> 1 : lane] = l[0];
        sync_unit();
        // a stream without a tile here has seen nothing
        if (leads && key < n_rows) {
          const float s_self = s_self_of[key];
          float l2[2], m2[2];
          for (int s = 0; s < 2; ++s) {
            const bool seen = (!alone || s == stream) && !sm.unseen[s][key];
            l2[s] = !alone || s == stream ? (sm.red[s][0][key] + sm.red[s][1][key]) + (sm.red[s][2][key] + sm.red[s][3][key]) : 0.0f;
            m2[s] = seen ? sm.m[s][key] : -INFINITY;
          }
          const float m0 = m2[0], m1 = m2[1];
          const float top = fmaxf(fmaxf(m0, m1), s_self);
          const float f0 = m0 == -INFINITY ? 0.0f : ex2_approx(m0 - top), f1 = m1 == -INFINITY ? 0.0f : ex2_approx(m1 - top);
          const float p_self = s_self == -INFINITY ? 0.0f : ex2_approx(s_self - top);
          // (NaN scores leave the references alone: they are in the sums)
          float sum = fmaf(f0, l2[0], fmaf(f1, l2[1], p_self));
          if (l2[0] != l2[0] || l2[1] != l2[1]) sum = l2[0] + l2[1];
          if (s_self != s_self) sum = s_self;
          const bool bad = alone ? sm.bad[stream][key] != 0 : (sm.bad[0][key] | sm.bad[1][key]) != 0;
          fin[key] = make_float4(f0, f1, p_self, bad ? kNan : place != -1 ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum);
          if (place == -2) sm.ml[key] = make_float2(top, sum);
          else if (place >= 0) p.part_ml[static_cast<size_t>(place) * kN + key] = make_float2(top, sum);
          else if (p.lse != nullptr) p.lse[orow0 + key] = (top + lg2_approx(sum)) * 0.6931471805599453f;
        }
        sync_unit();
        // thread = output column; the streams' warps take four rows in turn. Whose accumulators hold products of this unit: with two tiles and more
        // both streams', else the tile's (g is the one behind it).
        const bool has0 = alone ? stream == 0 : nt > 1 || (g & 1) == 1, has1 = alone ? stream == 1 : nt > 1 || (g & 1) == 0;
#pragma unroll 1
        for (int c0 = alone ? 0 : 4 * stream; c0 < n_rows; c0 += alone ? 4 : 8) {
          uint32_t o[2][4];
          tmem_ld4(quad + 2 * kN + c0, o[0]);
          tmem_ld4(quad + 3 * kN + c0, o[1]);
          tmem_ld_wait4(o[0]);
          tmem_ld_wait4(o[1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = c0 + e;
            if (i >= n_rows) break;
            const float4 f = fin[i];
            // (a weight of zero counts too: a value that is not finite makes its column NaN there)
            float x = has0 ? __uint_as_float(o[0][e]) * f.x : 0.0f;
            if (has1) x = fmaf(__uint_as_float(o[1][e]), f.y, x);
            if (own_rows) {
              const int4 row = sm.row[buf][i];
              if (row.z >= 0) x = fmaf(f.z, __bfloat162float(p.v_seedmask[(masked0 + row.w) * kD + key]), x);
            }
            x *= f.w;
            if (place == -2) sts32(staged + staged_at(i, key >> 2) + 4 * (key & 3), __float_as_uint(x));
            else if (place >= 0) p.part_o[(static_cast<size_t>(place) * kN + i) * kD + key] = x;
            else p.out[(orow0 + i) * kD + key] = __float2bfloat16_rn(x);
          }
          __syncwarp();
        }
      }
      tc_fence_before_sync();
      // both accumulators have been read before a stream lets the next unit's products begin
      if (any_of<256>(1, !ok)) {
        ok = false;
        break;
      }
      if (lane == 0) mbar_arrive(&sm.unit_empty[first_unit % kUnits]);
      if (lane == 0 && two) mbar_arrive(&sm.unit_empty[(first_unit + 1) % kUnits]);
      first_unit += two ? 2 : 1;
    }
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 84);
      sm.abort = 1;
    }
    tc_fence_before_sync();
    if (kJoined) {
      const int u = static_cast<int>(blockIdx.x) / p.joined % heads, p0 = u % p.n_groups * kN;
      __syncwarp();
      cluster_sync();   // every CTA's rows are staged
      join_rows<8>(p, staged, smem_u32(sm.ml), min(kN, n_packed - p0),
                   (static_cast<long long>(b0) * p.Hq + (u / p.n_groups) * p.G) * p.Lq + p0, static_cast<int>(blockIdx.x % p.joined), p.joined);
      __syncwarp();
      cluster_sync();   // no CTA leaves while its rows are read
    }
  }
  if (kJoined && warp >= kScreenWarp) join_pass();
  __syncthreads();
  if (warp == kRowsMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, kTmem);
  }
}

// Adds up the parts of a unit that began in main CTA blockIdx.y: a warp a row, four columns a lane.
constexpr int kJoinWarps = 4;
template <int kN>
__global__ void __launch_bounds__(kJoinWarps * 32) attn_paged_join_rows_kernel(const __grid_constant__ Params p) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, i = blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  const int4 join = p.joins[blockIdx.y];   // parts, rows, first row
  if (i >= join.y) return;
  // the first part is the last of its CTA, the others the first of theirs
  const auto at = [&](int k) { return (2 * (static_cast<size_t>(blockIdx.y) + k) + (k == 0 ? 1 : 0)) * kN + i; };
  float m = -INFINITY;
  for (int k = lane; k < join.x; k += 32) m = fmaxf(m, p.part_ml[at(k)].x);
  for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  float l = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int k = 0; k < join.x; ++k) {
    const float2 ml = p.part_ml[at(k)];
    const float4 o = *reinterpret_cast<const float4*>(p.part_o + at(k) * kD + 4 * lane);
    const float w = ml.x == -INFINITY ? 0.0f : ex2_approx(ml.x - m);
    l = ml.x == -INFINITY ? l + ml.y : fmaf(w, ml.y, l);   // (a sum of NaN is taken along)
    acc.x = fmaf(w, o.x, acc.x), acc.y = fmaf(w, o.y, acc.y), acc.z = fmaf(w, o.z, acc.z), acc.w = fmaf(w, o.w, acc.w);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const long long row = static_cast<long long>(join.z) + i;
  reinterpret_cast<uint2*>(p.out + row * kD)[lane] =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (lane == 0 && p.lse != nullptr) p.lse[row] = (m + lg2_approx(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------
// Many rows
// ---------------------------------------------------------------------------
// A CTA takes two Q tiles of 128 packed rows, a stream each, that read each KV tile together, against one of nsplit parts of the keys that its
// rows see. Two threads of different warpgroups share a row, 64 columns each, in two chunks of 32.
// Roles (640 threads): warps 0-15 softmax (warpgroup 2 t + h: columns 64 h .. 64 h + 63 of Q tile t); 16 products; 17, 18 copies of K and V.
// The softmax warps look V tiles through.
// Shared memory: Q (2 x 32 KB) | two tiles of K, two of V. Tensor memory: S0 | S1 (the P of a half overwrites the first 32 columns of that
// half's scores, behind its loads) | O0 | O1, 128 columns each.
constexpr int kPairsThreads = 640;   // (the last warp has no part: with 19 warps 2048 rows over 8192 keys took 270 us, with 20 266)
constexpr int kPairSoftmaxWarps = 16, kPairMmaWarp = 16, kPairCopyWarp = 17;

struct PairSmem {
  uint8_t q[2][kTileBytes];
  uint8_t k[2][kTileBytes];
  uint8_t v[2][kTileBytes];
  uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], v_clean[2];
  uint64_t s_full[2], p_full[2], o_full, drain;
  uint4 nan_keys[4];                    // per KV tile in turn: keys whose V row is not finite
  float2 ml[2 * kBM];                   // joined in a cluster: the rows' references and sums
  float s_self[2 * kBM];                // and their own pairs' scores and slots
  int own_slot[2 * kBM];
  float red[2][2][kBM];                 // per Q tile and half of the columns
  int slot[2 * kBM];                    // seed slot of a row's position, or kNoSlot
  int lo, hi;                           // keys that some row sees
  int all_lo, all_hi;                   // keys that every row sees that sees any
  int own_lo, own_hi;                   // seed rows' positions
  uint32_t tmem_base;
  int abort;
};

// This part's KV tiles among those that the CTA's rows see.
__device__ __forceinline__ int2 part_of(int lo, int hi, int ks, int nsplit) {
  const int t0 = hi > 0 ? lo / kBN : 0, t1 = hi > 0 ? (hi - 1) / kBN + 1 : 0;
  const int each = (t1 - t0) / nsplit, more = (t1 - t0) % nsplit;
  return make_int2(t0 + ks * each + min(ks, more), each + (ks < more ? 1 : 0));
}

// What a row sees of 64 columns of a KV tile, a bit each, and whether some row of the warp does not see some
// column of the first or the second 32.
struct Seen {
  uint32_t first, second;
  bool some_first, some_second;
};

// Bits lo <= c < hi of 32.
__device__ __forceinline__ uint32_t bits_of(int lo, int hi) {
  const uint32_t below = hi >= 32 ? 0xffffffffu : hi <= 0 ? 0u : (1u << hi) - 1u;
  return lo <= 0 ? below : lo >= 32 ? 0u : below & ~((1u << lo) - 1u);
}

// Masks the scores of 32 columns: a bit a column (compared with a row's range and its own position one by one, in both passes over the
// scores, the columns took a KV tile from 1.6 to 3.6 us).
__device__ __forceinline__ void mask_scores(float (&s)[32], const Seen& u, int c0) {
  if (c0 == 0 ? u.some_first : u.some_second) {
    const uint32_t seen = c0 == 0 ? u.first : u.second;
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (!((seen >> c) & 1u)) s[c] = -INFINITY;
  }
}

// The largest of 32 columns' scores, neither scaled nor capped yet.
__device__ __forceinline__ float chunk_max(uint32_t addr, const Seen& u, int c0) {
  uint32_t raw[32];
  tmem_ld32(addr, raw);
  tmem_ld_wait(raw);
  float(&s)[32] = reinterpret_cast<float(&)[32]>(raw);
  mask_scores(s, u, c0);
  return max32(s);
}

// The weights of 32 columns whose scores less the reference, in log2 units, are s: in bf16 to tensor memory (V's operands are, so P's have to be: a
// weight is off by at most 2^-8 of itself). Returns their sum before rounding.
__device__ __forceinline__ float store_weights(float (&s)[32], uint32_t p_addr, const Seen& u, int c0) {
  mask_scores(s, u, c0);
  uint64_t acc2[2] = {0, 0};
  uint32_t packed[16];
#pragma unroll
  for (int c = 0; c < 16; ++c) {
    const float e0 = ex2_approx(s[2 * c]), e1 = ex2_approx(s[2 * c + 1]);
    packed[c] = pack_bf16x2(e0, e1);
    acc2[c & 1] = f2_add(acc2[c & 1], f2_pack(e0, e1));
  }
  tmem_st16(p_addr, packed);
  float r[4];
  f2_unpack(acc2[0], r[0], r[1]);
  f2_unpack(acc2[1], r[2], r[3]);
  return (r[0] + r[1]) + (r[2] + r[3]);
}

// chunk_exp where some score is beyond the polynomial's range (kept out of the loop's code).
__device__ __noinline__ float chunk_exp_far(uint32_t addr, uint32_t p_addr, float cap_in, float cap_log2, const Seen u, int c0, float m) {
  uint32_t raw[32];
  tmem_ld32(addr, raw);
  tmem_ld_wait(raw);
  float(&s)[32] = reinterpret_cast<float(&)[32]>(raw);
#pragma unroll
  for (int e = 0; e < 32; ++e) s[e] = capped(s[e], cap_in, cap_log2) - m;
  return store_weights(s, p_addr, u, c0);
}

// P = 2^(score - m) of 32 columns to tensor memory; returns the sum of the unrounded weights. Capped scores of a chunk that are all within the
// polynomial's range take it, x P(x^2) with the scale's powers in its coefficients, and no special function (with three of them a score a KV
// tile took 3.2 us).
template <bool kCap>
__device__ __forceinline__ float chunk_exp(uint32_t addr, uint32_t p_addr, const Params& p, const Seen& u, int c0, float m, bool valid) {
  uint32_t raw[32];
  tmem_ld32(addr, raw);
  tmem_ld_wait(raw);
  float(&s)[32] = reinterpret_cast<float(&)[32]>(raw);
  const uint64_t negm2 = f2_pack(-m, -m);
  if (!kCap) {
    const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2);
#pragma unroll
    for (int e = 0; e < 32; e += 2) f2_unpack(f2_fma(f2_pack(s[e], s[e + 1]), scale2, negm2), s[e], s[e + 1]);
  } else {
    float hi[2] = {};
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      hi[0] = fmax3(hi[0], fabsf(s[c]), fabsf(s[c + 1]));
      hi[1] = fmax3(hi[1], fabsf(s[c + 2]), fabsf(s[c + 3]));
    }
    if (__any_sync(0xffffffffu, valid && !(fmaxf(hi[0], hi[1]) <= p.cap_near))) return chunk_exp_far(addr, p_addr, p.cap_in, p.cap_log2, u, c0, m);
    const uint64_t t0 = f2_pack(p.cap_poly[0], p.cap_poly[0]), t1 = f2_pack(p.cap_poly[1], p.cap_poly[1]),
                   t2 = f2_pack(p.cap_poly[2], p.cap_poly[2]), t3 = f2_pack(p.cap_poly[3], p.cap_poly[3]);
#pragma unroll
    for (int e = 0; e < 32; e += 2) {   // (a NaN among the scores stays one)
      const uint64_t x = f2_pack(s[e], s[e + 1]), z = f2_mul(x, x);
      f2_unpack(f2_fma(x, f2_fma(z, f2_fma(z, f2_fma(z, t3, t2), t1), t0), negm2), s[e], s[e + 1]);
    }
  }
  return store_weights(s, p_addr, u, c0);
}

// 64 columns' share of a seed row's own product: q from its half of a swizzled Q tile (row R), the masked-input key from global memory.
__device__ __forceinline__ float self_product(const uint8_t* q_half, int R, const __nv_bfloat16* k) {
  const uint32_t q = smem_u32(q_half) + R * 128;
  uint4 c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __ldg(reinterpret_cast<const uint4*>(k) + i);
  float d0 = 0.0f, d1 = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 a = lds128(q + ((i ^ (R & 7)) << 4));
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      d0 = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), d0);
      d1 = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), d1);
    }
  }
  return d0 + d1;
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

template <bool kCap>
__global__ void __launch_bounds__(kPairsThreads, 1)
    attn_paged_pairs_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                            const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  PairSmem& sm = *reinterpret_cast<PairSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // CTA (ks, hkv, group, b). A sequence's last rows see the most keys where they see what is before them, so they come first: the CTAs
  // that are left for the end are short ones (2048 rows over 8192 keys, blocks, 256 CTAs on 152 SMs: 225 us in the heads' order, 218 so).
  const int ks = static_cast<int>(blockIdx.x) % p.nsplit;
  int rest = static_cast<int>(blockIdx.x) / p.nsplit;
  const int hkv = rest % p.Hkv;
  rest /= p.Hkv;
  const int group = p.n_groups - 1 - rest % p.n_groups;
  const int b = rest / p.n_groups;
  const int n_packed = p.G * p.Lq;
  const int p0 = group * 2 * kBM;
  const long long rowbase = (static_cast<long long>(b) * p.Hq + hkv * p.G) * p.Lq;

  if (warp == kPairMmaWarp) {
    if (lane == 0) {
      mbar_init(&sm.q_full, 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.k_full[i], 1);
        mbar_init(&sm.k_empty[i], 1);
        mbar_init(&sm.v_full[i], 1);
        mbar_init(&sm.v_empty[i], 1);
        mbar_init(&sm.v_clean[i], p0 + kBM < n_packed ? kPairSoftmaxWarps : kPairSoftmaxWarps / 2);
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], 256);
      }
      sm.all_lo = 0;
      sm.all_hi = 0x7fffffff;
      mbar_init(&sm.o_full, 1);
      mbar_init(&sm.drain, 1);
      sm.abort = 0;
      sm.lo = 0x7fffffff;
      sm.hi = 0;
      sm.own_lo = 0x7fffffff;
      sm.own_hi = -1;
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
  const int tile = warp >> 3, half = (warp >> 2) & 1;   // of a softmax warp
  const int R = tid & (kBM - 1);
  const int P = p0 + tile * kBM + R;
  const bool softmax = warp < kPairSoftmaxWarps;
  const bool valid = softmax && P < n_packed;
  const int r = valid ? P % p.Lq : 0;
  constexpr int kKnowing = 32 * kPairSoftmaxWarps;   // the softmax warps' threads
  // loads that depend on nothing first: the sequence's first position and a seed, the table, the length
  int first_pos = 0, first_seed = 0;
  if (p.n_seeds > 0) {
    first_pos = __ldg(p.q0 + b);
    if (tid < p.n_seeds) first_seed = __ldg(p.seed_idx + static_cast<size_t>(b) * p.n_seeds + tid);
  }
  int line = 0;
  if (warp == kPairCopyWarp && lane * 32 < p.M)   // the table's first lines are on their way to L1 while the length is
    asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(line) : "l"(p.table + static_cast<size_t>(b) * p.M + lane * 32));
  const int len = length_of(p, b);
  asm volatile("" ::"r"(line));
  int row_lo = 0, row_hi = 0;
  if (valid) {
    const int2 keys = keys_of(p, static_cast<long long>(b) * p.Lq + r, len);
    row_lo = keys.x, row_hi = keys.y;
  }
  const bool some_keys = row_lo < row_hi;
  int lo_key = 0, hi_key = len;   // keys that some row sees
  if (p.key_lo != nullptr || p.key_hi != nullptr) {
    if (softmax) {
      const int lo = __reduce_min_sync(0xffffffffu, some_keys ? row_lo : 0x7fffffff), hi = __reduce_max_sync(0xffffffffu, row_hi);
      if (lane == 0 && hi > 0) {
        atomicMin(&sm.lo, lo);
        atomicMax(&sm.hi, hi);
      }
    }
    __syncthreads();
    lo_key = sm.lo, hi_key = sm.hi;
  }
  const int2 part = part_of(lo_key, hi_key, ks, p.nsplit);
  const int j0 = part.x, nt = part.y;
  const int page_rows = min(p.page_log2, 7), pages = kBN >> page_rows;   // of a KV tile
  const bool two_tiles = p0 + kBM < n_packed;   // the second Q tile has rows
  // What the softmax warps have to know besides; copies and products do not wait for it.
  int slot = kNoSlot, pos = -1;   // of a seed row that sees its position
  bool holes = false;             // some page with keys that rows see is not there
  if (softmax) {
    if (p.n_seeds > 0) {
      // the CTA's rows stand at up to 256 positions: r itself, or r - r0 around Lq
      const int r0 = p.Lq <= 2 * kBM ? 0 : p0 % p.Lq;
      const int32_t* seeds = p.seed_idx + static_cast<size_t>(b) * p.n_seeds;
      const int own_at = position_of(first_pos, r);
      const bool own = valid && own_at >= row_lo && own_at < row_hi;   // the row sees its position, if it has a page
      const int own_page = own ? page_of(p, b, own_at) : -1;
      for (int s = tid; s < p.n_seeds; s += kKnowing) {
        const long long at = static_cast<long long>(s == tid ? first_seed : __ldg(seeds + s)) - first_pos;
        if (at < 0 || at >= p.Lq) continue;
        const long long i = at >= r0 ? at - r0 : at - r0 + p.Lq;
        if (i < 2 * kBM) atomicMin(&sm.slot[i], s);
      }
      sync_of<kKnowing>(1);
      if (own_page >= 0) {
        slot = sm.slot[r >= r0 ? r - r0 : r - r0 + p.Lq];
        if (slot != kNoSlot) pos = own_at;
      }
    }
    const int all_lo = __reduce_max_sync(0xffffffffu, row_lo), all_hi = __reduce_min_sync(0xffffffffu, some_keys ? row_hi : 0x7fffffff);
    const int own_lo = __reduce_min_sync(0xffffffffu, slot != kNoSlot ? pos : 0x7fffffff), own_hi = __reduce_max_sync(0xffffffffu, pos);
    if (lane == 0) {
      atomicMax(&sm.all_lo, all_lo);
      atomicMin(&sm.all_hi, all_hi);
      if (own_hi >= 0) atomicMin(&sm.own_lo, own_lo), atomicMax(&sm.own_hi, own_hi);
    }
    bool hole = false;
    for (int i = tid; i < nt * pages; i += kKnowing) {
      const int key = j0 * kBN + (i << page_rows);
      if (key < hi_key && lo_key - key < 1 << page_rows) hole |= page_of(p, b, key) < 0;
    }
    holes = any_of<kKnowing>(1, hole);
  }
  const bool is_seed = slot != kNoSlot;
  // whether some row that sees a key does not see some key of KV tile j of the part
  const int all_lo = sm.all_lo, all_hi = sm.all_hi, own_lo = sm.own_lo, own_hi = sm.own_hi;
  const auto partial = [&](int j) {
    const int key0 = (j0 + j) * kBN;
    return holes || key0 < all_lo || all_hi - key0 < kBN || (own_hi >= key0 && own_lo - key0 < kBN);
  };

  if (warp >= kPairMmaWarp) {
    if (warp == kPairMmaWarp && lane == 0 && nt > 0) {
      // ---------------- products ----------------
      constexpr uint32_t id_qk = idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t id_pv = idesc_bf16_f32(kBM, kD, false, true);
      constexpr uint32_t kTileDesc = kTileBytes >> 4;
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[0]), 16, 1024);
      const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, kGroupBytes);
      const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), kGroupHalf, kGroupBytes);
      // descriptors are added up in their lower words, and of several barriers the one that completes last is waited for last: what
      // this thread does between a barrier and its products is on every tile's way
      const uint32_t q_lo = static_cast<uint32_t>(dq), k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv);
      const uint32_t q_hi = static_cast<uint32_t>(dq >> 32), kv_hi = static_cast<uint32_t>(dk >> 32);
      const auto desc = [](uint32_t lo, uint32_t hi) { return (static_cast<uint64_t>(hi) << 32) | lo; };
      // S[s] = Q[s] . K(stage)^T
      auto issue_s = [&](int s, int st) {
        const uint32_t a = q_lo + s * kTileDesc, kb = k_lo + st * kTileDesc;
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          umma_ss(tbase + s * kBN, desc(a + (((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4), q_hi),
                  desc(kb + (((kk >> 2) * kGroupHalf + (kk & 3) * 32) >> 4), kv_hi), id_qk, kk > 0 ? 1u : 0u);
        }
        umma_commit(&sm.s_full[s]);
      };
      // O[s] (+)= P[s] . V(stage)
      auto issue_pv = [&](int s, int st, bool acc) {
        const uint32_t vb = v_lo + st * kTileDesc;
#pragma unroll
        for (int kk = 0; kk < kBN / 16; ++kk)
          umma_ts(tbase + 2 * kBN + s * kD, tbase + s * kBN + (kk >> 2) * kHalf + 8 * (kk & 3),
                  desc(vb + ((kk * 2 * kGroupBytes) >> 4), kv_hi), id_pv, (acc || kk > 0) ? 1u : 0u);
      };
      auto wait = [&](uint64_t* bar, int phase) {
        const bool ok = mbar_wait(bar, phase & 1, &sm.abort);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      bool ok = wait(&sm.q_full, 0);
      if (ok && (ok = wait(&sm.k_full[0], 0))) {
        issue_s(0, 0);
        if (two_tiles) issue_s(1, 0);
        umma_commit(&sm.k_empty[0]);
      }
      for (int j = 0; j < nt && ok; ++j) {
        const int st = j & 1;
        const bool next = j + 1 < nt;
        ok = (!next || wait(&sm.k_full[st ^ 1], (j + 1) >> 1)) && wait(&sm.v_full[st], j >> 1) && wait(&sm.v_clean[st], j >> 1) &&
             wait(&sm.p_full[0], j);
        if (!ok) break;
        issue_pv(0, st, j > 0);
        if (next) issue_s(0, st ^ 1);
        if (two_tiles) {
          ok = wait(&sm.p_full[1], j);
          if (!ok) break;
          issue_pv(1, st, j > 0);
          if (next) issue_s(1, st ^ 1);
        }
        umma_commit(&sm.v_empty[st]);
        if (next) umma_commit(&sm.k_empty[st ^ 1]);
      }
      if (ok) {
        umma_commit(&sm.o_full);
      } else {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 85);
        sm.abort = 1;
      }
      // all tensor-core work of this CTA completes before tensor memory is released
      umma_commit(&sm.drain);
      mbar_wait(&sm.drain, 0, nullptr);
    } else if ((warp == kPairCopyWarp || warp == kPairCopyWarp + 1) && nt > 0) {
      // ---------------- copies ----------------
      const int which = warp - kPairCopyWarp;
      const CUtensorMap* tm = which ? &tm_v : &tm_k;
      uint64_t* const full = which ? sm.v_full : sm.k_full;
      uint64_t* const empty = which ? sm.v_empty : sm.k_empty;
      if (which == 0 && lane == 0) {
        mbar_arrive_expect_tx(&sm.q_full, 2 * kTileBytes);
        for (int t = 0; t < 2; ++t)
          for (int h = 0; h < 2; ++h)
            tma_load_4d(sm.q[t] + h * kBoxBytes, &tm_q, &sm.q_full, 64 * h, static_cast<int>(rowbase) + p0 + t * kBM, 0, 0);
      }
      // a lane's page of the next tile is looked up a tile ahead
      const int my_key = (lane % pages) << page_rows;
      int entry = page_of(p, b, j0 * kBN + my_key);
      int j = 0;
      bool ok = true;
      for (; j < nt; ++j) {
        const int st = j & 1;
        const int next = j + 1 < nt ? page_of(p, b, (j0 + j + 1) * kBN + my_key) : -1;
        if (j >= 2) ok = warp_wait(&empty[st], ((j >> 1) - 1) & 1, &sm.abort);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&full[st], kTileBytes);
        __syncwarp();
        copy_tile(tm, which ? sm.v[st] : sm.k[st], &full[st], (j0 + j) * kBN, entry, hkv, p.Hkv, p.page_log2, lane);
        __syncwarp();
        entry = next;
      }
      if (!ok && lane == 0) {
        if (!sm.abort) report_status(p.status, kStatusTimeout, 86);
        sm.abort = 1;
      }
      // every copy lands before the CTA's shared memory is released, whatever the other roles did
      if (lane == 0) {
        if (which == 0) mbar_wait(&sm.q_full, 0, nullptr);
        for (int f = max(0, j - 2); f < j; ++f) mbar_wait(&full[f & 1], (f >> 1) & 1, nullptr);
      }
    }
    __syncwarp();
  } else {
    // ---------------- softmax ----------------
    const size_t self = (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds + (is_seed ? slot : 0);
    const bool own_here = own_hi >= 0 && ks == 0;   // the seed rows' own pairs are added in the first part of the keys
    if (own_here && is_seed) {
      prefetch_l2(p.k_seedmask + self * kD + half * kHalf);
      prefetch_l2(p.v_seedmask + self * kD + half * kHalf);
    }
    bool ok = true;
    const bool warp_live = __any_sync(0xffffffffu, valid);
    const uint32_t quad = tbase + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = quad + tile * kBN + half * kHalf;
    const uint32_t o_addr = quad + 2 * kBN + tile * kD + half * kHalf;
    const bool fixed = kCap && p.cap_ref >= 0.0f;
    float m_run = fixed ? p.cap_ref : -INFINITY, l_run = 0.0f;
    const int jend = tile == 1 && !two_tiles ? 0 : nt;
    // Where some row does not see some key, V is looked through for rows that are not finite while the scores are waited for: a warp eight
    // keys, or sixteen (a warp for all of it took a tile 1.5 us). What was found is read a tile later.
    bool bad = false;   // the row sees a V row that was set to zeros
    const auto found = [&](int j) {
      if (!warp_wait(&sm.v_clean[j & 1], (j >> 1) & 1, &sm.abort)) {
        ok = false;
        return;
      }
      // a row that sees one of these keys is NaN (both threads of it look, for all 128)
      const uint4 nan = sm.nan_keys[j & 3];
      if ((nan.x | nan.y | nan.z | nan.w) == 0) return;
#pragma unroll 1
      for (int w = 0; w < 4; ++w) {
        for (uint32_t bits = w == 0 ? nan.x : w == 1 ? nan.y : w == 2 ? nan.z : nan.w; bits != 0; bits &= bits - 1) {
          const int at = (j0 + j) * kBN + 32 * w + __ffs(bits) - 1;
          bad |= at >= row_lo && at < row_hi && !(is_seed && at == pos);
        }
      }
    };
    const bool keyless = __any_sync(0xffffffffu, valid && !some_keys);   // a row of the warp sees no key at all
    bool masked = false;
    for (int j = 0; j < jend; ++j) {
      const int key0 = (j0 + j) * kBN + half * kHalf;
      if (masked) found(j - 1);
      masked = partial(j);
      Seen u{0xffffffffu, 0xffffffffu, false, false};
      bool some = warp_live;   // a warp none of whose rows sees a key here stores zeros; a row without a query row may hold anything
      if (masked) {
        ok = warp_wait(&sm.v_full[j & 1], (j >> 1) & 1, &sm.abort) && ok;   // (its copy waits for the products of tile j - 2 alone)
        if (ok)
          for (int g = warp; g < kBN / 8; g += two_tiles ? kPairSoftmaxWarps : kPairSoftmaxWarps / 2)
            screen_group(smem_u32(sm.v[j & 1]) + g * kGroupBytes, reinterpret_cast<uint8_t*>(&sm.nan_keys[j & 3]) + g, lane);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.v_clean[j & 1]);
      if (masked || keyless) {
        const int cl = row_lo - key0, ch = row_hi - key0;   // columns cl <= c < ch of this half are seen
        u.first = bits_of(cl, ch);
        u.second = bits_of(cl - 32, ch - 32);
        if (is_seed && pos - key0 >= 0 && pos - key0 < kHalf) {
          const uint32_t own = ~(1u << (pos & 31));
          if (pos - key0 < 32) u.first &= own;
          else u.second &= own;
        }
        if (holes) {
          const uint32_t there = __ballot_sync(0xffffffffu, page_of(p, b, key0 + 2 * lane) >= 0);   // two keys a lane
          // pages are of 16 keys at least: eight lanes'
          u.first &= ((there & 0xffu) != 0 ? 0xffffu : 0u) | ((there & 0xff00u) != 0 ? 0xffff0000u : 0u);
          u.second &= ((there & 0xff0000u) != 0 ? 0xffffu : 0u) | ((there & 0xff000000u) != 0 ? 0xffff0000u : 0u);
        }
        u.some_first = __any_sync(0xffffffffu, valid && u.first != 0xffffffffu);
        u.some_second = __any_sync(0xffffffffu, valid && u.second != 0xffffffffu);
        some = __any_sync(0xffffffffu, valid && (u.first | u.second) != 0);
      }
      ok = warp_wait(&sm.s_full[tile], j & 1, &sm.abort) && ok;
      tc_fence_after_sync();   // zeros are stored over S too, where no row sees a key
      if (fixed) {
        if (!ok) break;
      } else {
        float m_half = -INFINITY;
        if (ok && some) {
#pragma unroll 1
          for (int c = 0; c < kHalf; c += 32) m_half = fmaxf(m_half, chunk_max(s_addr + c, u, c));
          m_half = !kCap ? m_half * p.scale_log2 : m_half == -INFINITY ? m_half : capped(m_half, p.cap_in, p.cap_log2);   // (the cap is monotonous)
        }
        // The Q tile's 256 threads vote: a warp whose wait gave up takes part all the same, and both halves of a row
        // take the same reference
        if (any_of<256>(2 + tile, !ok || (valid && m_half > m_run + kRescaleThreshold))) {
          if (any_of<256>(2 + tile, !ok)) {
            ok = false;
            break;
          }
          sm.red[tile][half][R] = m_half;
          sync_of<256>(2 + tile);
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
      }
      if (some) {
        const float m_use = (m_run == -INFINITY) ? 0.0f : m_run;
#pragma unroll 1
        for (int c = 0; c < kHalf; c += 32) l_run += chunk_exp<kCap>(s_addr + c, s_addr + c / 2, p, u, c, m_use, valid);
      } else if (warp_live) {
        const uint32_t zeros[16] = {};
        tmem_st16(s_addr, zeros);
        tmem_st16(s_addr + 16, zeros);
      }
      tmem_st_wait();
      tc_fence_before_sync();
      mbar_arrive(&sm.p_full[tile]);
    }
    // Their scores (log2 units), while V's last products are on their way: Q is still there, and each of a row's threads takes half of the
    // columns. (Before the first scores, 32 rows over 1024 keys with 32 seeds took 0.5 us more.)
    float s_self = -INFINITY;
    if (own_here) {
      float product = 0.0f;
      ok = ok && (nt == 0 || warp_wait(&sm.q_full, 0, &sm.abort));
      if (ok && nt > 0 && is_seed) product = self_product(sm.q[tile] + half * kBoxBytes, R, p.k_seedmask + self * kD + half * kHalf);
      sync_of<256>(2 + tile);   // the last references have been read
      sm.red[tile][half][R] = product;
      sync_of<256>(2 + tile);
      if (is_seed) {
        const float s = sm.red[tile][0][R] + sm.red[tile][1][R];
        s_self = kCap ? capped(s, p.cap_in, p.cap_log2) : s * p.scale_log2;
      }
      if (p.joined) sync_of<kKnowing>(1);   // a tile's results are staged where the other tile's Q is
    }
    if (ok && nt > 0) ok = warp_wait(&sm.o_full, 0, &sm.abort);
    if (ok && masked) found(jend - 1);
    if (!ok && lane == 0) {
      if (!sm.abort) report_status(p.status, kStatusTimeout, 88);
      sm.abort = 1;
    }

    // ---------------- the rows' results ----------------
    tc_fence_after_sync();
    sync_of<256>(2 + tile);                     // the last references have been read
    sm.red[tile][half][R] = l_run;
    sync_of<256>(2 + tile);
    float m = m_run, l = sm.red[tile][0][R] + sm.red[tile][1][R], w = 1.0f, p_self = 0.0f;
    if (l == 0.0f) m = -INFINITY;               // no key was seen
    if (s_self != -INFINITY && !p.joined) {
      const float m_all = fmaxf(m, s_self);
      const float f = m == -INFINITY ? 0.0f : ex2_approx(m - m_all);
      p_self = ex2_approx(s_self - m_all);
      l = l * f + p_self;
      w = f;
      m = m_all;
    }
    if (s_self != s_self && !p.joined) l = s_self;   // NaN in the masked-input pair
    if (p.joined && half == 0) sm.s_self[tile * kBM + R] = s_self, sm.own_slot[tile * kBM + R] = slot;
    const long long orow = rowbase + P;
    const bool split = p.nsplit > 1;
    const float inv = split ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);   // 1 / l, once a row; zero where no key was seen
    if (bad) w = kNan;
    const uint32_t staged = smem_u32(sm.q[0]);   // joined: every product is complete, Q and K are not read any more
    // A warp's 32 rows of 128 bytes are turned in shared memory, where Q was, so that it stores whole lines (each thread its own row, 16 bytes
    // at a time: 3.6 us a CTA).
    const uint32_t turned = staged + warp * 4096 + lane * 128;
    const auto store_turned = [&](uint8_t* dst, int row_bytes) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = 4 * i + (lane >> 3), at = P - lane + row;
        const uint4 x = lds128(staged + warp * 4096 + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
        if (at < n_packed) *reinterpret_cast<uint4*>(dst + static_cast<long long>(at) * row_bytes + 16 * (lane & 7)) = x;
      }
    };
    if (ok && warp_live) {
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        float o[32] = {};
        if (nt > 0) {
          uint32_t x[32];
          tmem_ld32(o_addr + 32 * c, x);
          tmem_ld_wait(x);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = some_keys ? __uint_as_float(x[e]) * w : 0.0f;   // (what a row without keys has here may be NaN)
        }
        const int col = half * kHalf + 32 * c;
        if (own_here && is_seed && !p.joined) add_self(o, p_self, p.v_seedmask + self * kD + col);
        if (p.joined) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sts128(staged + staged_at(tile * kBM + R, col / 4 + e), __float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]),
                   __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3]));
        } else if (split) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sts128(turned + ((e ^ (lane & 7)) << 4), __float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]), __float_as_uint(o[4 * e + 2]),
                   __float_as_uint(o[4 * e + 3]));
          store_turned(reinterpret_cast<uint8_t*>(p.part_o + (static_cast<size_t>(ks) * p.rows + rowbase) * kD + col), kD * 4);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sts128(turned + (((4 * c + e) ^ (lane & 7)) << 4), pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv),
                   pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv), pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv),
                   pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
          if (c == 1) store_turned(reinterpret_cast<uint8_t*>(p.out + rowbase * kD + half * kHalf), kD * 2);
        }
        __syncwarp();   // the next chunk is loaded by the whole warp
      }
      if (valid && half == 0) {
        if (p.joined) sm.ml[tile * kBM + R] = make_float2(m, l);
        else if (split) p.part_ml[static_cast<size_t>(ks) * p.rows + orow] = make_float2(m, l);
        else if (p.lse != nullptr) p.lse[orow] = (m + lg2_approx(l)) * 0.6931471805599453f;
      }
    }
    tc_fence_before_sync();
    if (p.joined) {
      __syncwarp();
      cluster_sync();   // every CTA's rows are staged
      // the seed rows' own pairs are added with the parts (by the first CTA alone they held the others up for 1.1 us)
      join_rows<kPairSoftmaxWarps>(p, staged, smem_u32(sm.ml), min(2 * kBM, n_packed - p0), rowbase + p0, ks, p.nsplit,
                                   p.n_seeds > 0 ? sm.own_slot : nullptr, smem_u32(sm.s_self),
                                   p.v_seedmask + (static_cast<size_t>(b) * p.Hkv + hkv) * p.n_seeds * kD);
      __syncwarp();
      cluster_sync();   // no CTA leaves while its rows are read
    }
  }
  if (p.joined && warp >= kPairMmaWarp) join_pass();
  __syncthreads();
  if (warp == kPairMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tbase, 512);
  }
}

// Adds up the parts of every row: a warp a row, four columns a lane.
__global__ void __launch_bounds__(kJoinWarps * 32) attn_paged_join_pairs_kernel(const __grid_constant__ Params p) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kJoinWarps + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  float m = -INFINITY;
  for (int k = lane; k < p.nsplit; k += 32) m = fmaxf(m, p.part_ml[row + k * p.rows].x);
  for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  float l = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int k = 0; k < p.nsplit; ++k) {
    const float2 ml = p.part_ml[row + k * p.rows];
    const float4 o = *reinterpret_cast<const float4*>(p.part_o + (row + k * p.rows) * kD + 4 * lane);
    const float w = ml.x == -INFINITY ? 0.0f : ex2_approx(ml.x - m);
    l = ml.x == -INFINITY ? l + ml.y : fmaf(w, ml.y, l);   // (a sum of NaN is taken along)
    acc.x = fmaf(w, o.x, acc.x), acc.y = fmaf(w, o.y, acc.y), acc.z = fmaf(w, o.z, acc.z), acc.w = fmaf(w, o.w, acc.w);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  reinterpret_cast<uint2*>(p.out + row * kD)[lane] =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (lane == 0 && p.lse != nullptr) p.lse[row] = (m + lg2_approx(l)) * 0.6931471805599453f;
}

enum Mode { kRows16, kRows32, kPairs };

struct Plan {
  Mode mode;
  int n_groups, nsplit;
  int ctas;     // rows: of the main kernel, where its shares cross units
  int joined;   // CTAs of a cluster that share a unit, or 0
};

// Clusters of 1 .. 8 CTAs, one CTA an SM, that are resident at once on every GPU measured.
constexpr int kClusters[kMaxJoined] = {152, 76, 46, 36, 24, 20, 14, 14};

// The kernel and how the keys are shared, from the sizes and the table's width. The lengths are not known to the host, so the plan is that of
// sequences as long as the table is wide. Shorter ones are right by it, but another plan may be faster: with tables of 131072 positions one
// token over 777 keys takes 12.3 us (8.5 with a table of its length), 32 rows over 1024 with 32 seeds 24.4 (13.6), 2048 rows over 8192
// 304 (261) and 136 MB of workspace for four parts (none); a token of 64 sequences of up to 8191 keys 187 (186).
//
// Predicted microseconds, fitted to calls back to back on GB300, measured / predicted. Rows of 16 joined: one token over 777 keys (28 / 4 heads,
// 7 CTAs a unit) 7.6 / 7.7, over 4096 (32 / 8, 8) 12.0 / 11.8, 16 sequences of 500 (1) 12.8 / 13.3, 29 of 51 (1) 16.1 / 16.8. In even shares
// 11.5 / 13.0, 15.6 / 14.5, 18.8 / 17.0, 12.7 / 16.4; 128 sequences of 120 29.3 / 30.6, 256 of 100 48.2 / 49.7, 64 of 512 39.5 / 32.2. Rows of 32
// joined 12.6 / 13.0 (32 rows over 2048, 32 / 8), in even shares 8 sequences of 32 over 4000 44.6 / 38.7. Pairs joined: 8 rows over 2048
// (32 / 8, 8 CTAs a unit) 10.2 / 10.9, 8 sequences of 8 rows over 1000 (2) 15.6 / 16.6, 5 of 75 over 699 (16 / 2, 3) 15.3 / 16.9; by a second
// kernel 16.0 / 18.0; in one wave 18.5 / 18.1.
Plan plan_of(int B, int Hq, int Hkv, int Lq, int M, int page) {
  const long long packed = static_cast<long long>(Hq / Hkv) * Lq;
  const long long nkv = (static_cast<long long>(M) * page + kBN - 1) / kBN;   // KV tiles of a sequence at most
  const double rows = static_cast<double>(B) * Hq * Lq;
  Plan best{};
  double best_us = 0.0;
  const auto consider = [&](const Plan& plan, double us) {
    if (best.n_groups == 0 || us < best_us) best = plan, best_us = us;
  };
  if (packed <= 32) {
    const bool few = packed <= 16;
    const Mode mode = few ? kRows16 : kRows32;
    const long long units = static_cast<long long>(B) * Hkv;
    const double tile = few ? 1.48 : 2.2, fill = B > 1 && nkv > 1 ? 0.75 : 1.0;
    const int ctas = static_cast<int>(std::min<long long>(kSms, std::min<long long>(units, kSms) * std::min<long long>(nkv, kSms)));
    const double each = static_cast<double>(units) / kSms;
    consider(Plan{mode, 1, 1, ctas, 0}, (few ? 11.5 : 14.0) + tile * std::ceil(fill * each * nkv) + 1.3 * each);
    for (int c = 1; c <= kMaxJoined && c <= nkv; ++c) {
      const double waves = std::ceil(static_cast<double>(units) / kClusters[c - 1]);
      consider(Plan{mode, 1, 1, 0, c}, (few ? 6.3 : 9.8) + (units * c > kSms / 2 ? 1.5 : 0.0) + 6.2 * (waves - 1) +
                                           (few ? 1.38 : 1.6) * waves * std::ceil(static_cast<double>(nkv) / c));
    }
    if (few) return best;
  }
  const int groups = static_cast<int>((packed + 2 * kBM - 1) / (2 * kBM));
  const long long units = static_cast<long long>(groups) * Hkv * B;
  for (int ns = 1; ns <= nkv && ns <= 64; ++ns) {
    const double waves = std::ceil(static_cast<double>(units * ns) / kSms), tiles = std::ceil(static_cast<double>(nkv) / ns);
    consider(Plan{kPairs, groups, ns, 0, 0}, 5.0 + waves * (3.5 + 1.6 * tiles) + (ns > 1 ? 2.4 + 0.15 * ns + 1.9e-4 * rows * ns : 0.0));
    if (ns > 1 && ns <= kMaxJoined) {
      const double turns = std::ceil(static_cast<double>(units) / kClusters[ns - 1]);
      const double join = 4.0 * std::min<long long>(packed, 2 * kBM) / (2 * kBM);   // of a unit's rows
      consider(Plan{kPairs, groups, ns, 0, ns},
               7.2 + (units * ns > kSms / 2 ? 2.5 : 0.0) + 3.5 * (turns - 1) + turns * (1.6 * tiles + join));
    }
    if (units * ns > 8 * kSms) break;
  }
  return best;
}

constexpr size_t kRowsSmemBytes[2] = {sizeof(RowsSmem<16>) + 1024, sizeof(RowsSmem<32>) + 1024};
constexpr size_t kPairSmemBytes = sizeof(PairSmem) + 1024;
static_assert(kRowsSmemBytes[0] <= 227 * 1024 && kRowsSmemBytes[1] <= 227 * 1024 && kPairSmemBytes <= 227 * 1024, "shared memory of a CTA");

using Kernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const Params);
template <int kN>
constexpr Kernel kRowsOf[2][2] = {{attn_paged_rows_kernel<kN, false, false>, attn_paged_rows_kernel<kN, false, true>},
                                  {attn_paged_rows_kernel<kN, true, false>, attn_paged_rows_kernel<kN, true, true>}};
constexpr Kernel kPairKernels[2] = {attn_paged_pairs_kernel<false>, attn_paged_pairs_kernel<true>};

// rows of all parts
size_t part_rows(const Plan& plan, int B, int Hq, int Lq) {
  if (plan.joined) return 0;
  if (plan.mode != kPairs) return static_cast<size_t>(2 * plan.ctas) * (plan.mode == kRows16 ? 16 : 32);
  return plan.nsplit > 1 ? static_cast<size_t>(B) * Hq * Lq * plan.nsplit : 0;
}

// The plan of a debug call: `parts` parts of the keys or CTAs, negative: as many CTAs of a cluster.
Plan forced(int Hq, int Hkv, int Lq, int mode, int parts) {
  const long long packed = static_cast<long long>(Hq / Hkv) * Lq;
  const int width = mode == kPairs ? 2 * kBM : mode == kRows16 ? 16 : 32, joined = parts < 0 ? -parts : 0;
  return Plan{static_cast<Mode>(mode), static_cast<int>((packed + width - 1) / width), mode == kPairs ? std::abs(parts) : 1,
              mode == kPairs || joined ? 0 : parts, joined};
}

size_t plan_bytes(const Plan& plan, int B, int Hq, int Lq) {
  return part_rows(plan, B, Hq, Lq) * (kD * sizeof(float) + sizeof(float2)) + plan.ctas * sizeof(int4);
}

}  // namespace

size_t attn_paged_workspace_bytes(int B, int Hq, int Hkv, int Lq, int M, int page) {
  return plan_bytes(plan_of(B, Hq, Hkv, Lq, M, page), B, Hq, Lq);
}
size_t attn_paged_mode_bytes(int B, int Hq, int Hkv, int Lq, int mode, int parts) {
  return plan_bytes(forced(Hq, Hkv, Lq, mode, parts), B, Hq, Lq);
}

int launch_attn_paged(const AttnPagedArgs& a, int* status, cudaStream_t stream) {
  using bf16 = __nv_bfloat16;
  const Plan plan = a.mode >= 0 ? forced(a.Hq, a.Hkv, a.Lq, a.mode, a.parts) : plan_of(a.B, a.Hq, a.Hkv, a.Lq, a.M, a.page);
  const bool few = plan.mode != kPairs;
  const int width = plan.mode == kRows16 ? 16 : 32;
  const long long rows = static_cast<long long>(a.B) * a.Hq * a.Lq;
  const long long units = static_cast<long long>(plan.n_groups) * a.Hkv * a.B;
  const long long grid = plan.joined ? units * plan.joined : few ? plan.ctas : units * plan.nsplit;
  if (grid > 0x7fffffffLL) return -2;
  static ContextCache<int> setup;
  int unused = 0;
  const int rc = setup.get(&unused, [&](int&) {
    const auto limit = [](auto fn, size_t smem) {
      return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess;
    };
    for (int c = 0; c < 2; ++c) {
      for (int j = 0; j < 2; ++j)
        if (!limit(kRowsOf<16>[c][j], kRowsSmemBytes[0]) || !limit(kRowsOf<32>[c][j], kRowsSmemBytes[1])) return -3;
      if (!limit(kPairKernels[c], kPairSmemBytes)) return -3;
    }
    return 0;
  });
  if (rc != 0) return rc;
  CUtensorMap tq{}, tk{}, tv{};
  const uint32_t box = static_cast<uint32_t>(std::min(a.page, kBN)) / 8;
  const uint64_t groups = static_cast<uint64_t>(a.n_pages) * a.Hkv * a.page / 8;
  if (groups > 0x7fffffffULL) return -2;
  if (!make_bf16_map_4d(&tq, a.q, kD, static_cast<uint64_t>(rows), 1, 1, few ? width : kBM) ||
      !make_bf16_row_groups_map(&tk, a.k_pages, groups, box) || !make_bf16_row_groups_map(&tv, a.v_pages, groups, box))
    return -3;
  const float log2e = 1.4426950408889634f, root = sqrtf(static_cast<float>(kD));
  const bool cap = a.softcap > 0.0f;
  const float softcap = fminf(fmaxf(a.softcap, kMinCap), kMaxCap);
  Params p{};
  p.q = static_cast<const bf16*>(a.q);
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
  const size_t parts = part_rows(plan, a.B, a.Hq, a.Lq);
  p.part_o = static_cast<float*>(a.workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + parts * kD);
  p.joins = reinterpret_cast<int4*>(p.part_ml + parts);
  p.status = status;
  p.rows = rows;
  p.n_pages = a.n_pages;
  p.M = a.M;
  while ((1 << p.page_log2) < a.page) ++p.page_log2;
  p.B = a.B;
  p.n_seeds = a.n_seeds;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.Lq = a.Lq;
  p.n_groups = plan.n_groups;
  p.nsplit = plan.nsplit;
  p.joined = plan.joined;
  p.scale_log2 = log2e / root;
  p.cap_log2 = softcap * log2e;
  p.cap_in = cap ? 2.0f * log2e / (softcap * root) : 0.0f;
  // (caps below 2^-10 would put powers of 1 / cap beyond fp32's largest number)
  const float cap_x = cap ? 1.0f / (softcap * root) : 0.0f, tanh_poly[4] = {kTanh0, kTanh1, kTanh2, kTanh3};
  p.cap_ref = cap && p.cap_log2 <= kFixedCap ? fmaxf(0.0f, p.cap_log2 - kFixedRange) : -1.0f;
  p.cap_near = cap && p.cap_log2 >= 1.0f / 1024.0f ? kTanhRange / cap_x : -1.0f;
  float power = p.cap_log2 * cap_x;
  for (int i = 0; i < 4; ++i, power *= cap_x * cap_x) p.cap_poly[i] = p.cap_near > 0.0f ? tanh_poly[i] * power : 0.0f;
  cudaLaunchAttribute pdl[1], attr[2];
  const int m = plan.mode == kRows16 ? 0 : 1;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(few ? kRowsThreads : kPairsThreads),
                                      few ? kRowsSmemBytes[m] : kPairSmemBytes, stream, pdl);
  if (plan.joined) {
    attr[0] = pdl[0];
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(plan.joined);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
  const int joined = plan.joined > 0 ? 1 : 0, capped = cap ? 1 : 0;
  const Kernel kernel = !few ? kPairKernels[capped] : m == 0 ? kRowsOf<16>[capped][joined] : kRowsOf<32>[capped][joined];
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, tq, tk, tv, p);
  if (e == cudaSuccess && parts > 0) {
    const dim3 join_grid = few ? dim3(width / kJoinWarps, plan.ctas) : dim3(static_cast<unsigned>((rows + kJoinWarps - 1) / kJoinWarps));
    cfg = pdl_config(join_grid, dim3(kJoinWarps * 32), 0, stream, pdl);
    const auto join = !few ? attn_paged_join_pairs_kernel : m == 0 ? attn_paged_join_rows_kernel<16> : attn_paged_join_rows_kernel<32>;
    e = cudaLaunchKernelEx(&cfg, join, p);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? 0 : -3;
}

}  // namespace cover
