// kv8_kernel.cu - rows of keys and values into an 8-bit memory and back.
//
// The memory of a layer is k8, v8 [B, Hkv, L, D] e4m3 codes and k_exp, v_exp [B, Hkv, L] exponent bytes
// (e4m3.cuh). Slot s of a batch row stands for position pos0 + s, or pos[b, s] where a list is given.
//   write: x = the smallest byte with max |row| <= 448 * 2^(x - 127); code = the nearest e4m3 value of
//          row * 2^(127 - x). A listed position out of [0, L), or named by a lower slot of the same batch row
//          already, is left out (the lowest slot wins, as in the attention kernels' routing).
//   read:  row = code * 2^(x - 127); a position out of [0, L) gives zeros.
//
// Bound by memory: each row is read and written once. D / N lanes hold a row (N elements of 16 bytes on the wide
// side), and a thread has the K and V vectors of kTok = 2 consecutive slots in flight, 64 bytes, with six CTAs of 256
// threads an SM: 4 x 8 heads, 8191 rows of 128 bf16 from a projection are written in 35 us (with one slot and six
// CTAs 46, with four and four 42, eight and two 47, each with the positions taken from shared memory, where this took
// 37). A listed write loads its rows before it looks through the list: 8 x 32 heads, 64 rows of 64 fp32 5.2 us, and 5.8
// with the list first and a slot at a time.
#include <cuda_bf16.h>
#include <stdint.h>

#include <algorithm>

#include "e4m3.cuh"
#include "kernels.cuh"
#include "ptx.cuh"

namespace cover {
namespace {

constexpr int kThreads = 256;
constexpr int kTok = 2;   // slots of a lane group

struct Kv8Params {
  const uint8_t* src[2];     // k, v rows (write) or codes (read)
  uint8_t* dst[2];           // codes (write) or rows (read)
  uint8_t* exps[2];
  long long sb[2], sh[2], sl[2];   // strides of k, v in elements (write)
  const int32_t* pos;        // [B, n] or null
  int pos0, n, L, Hkv;
  int heads;                 // heads of a CTA
  int first;                 // of the grid's rows: tiles of slots written, or groups of heads read
};

template <typename T>
struct Wide;
template <>
struct Wide<__nv_bfloat16> {
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
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
  }
};
template <>
struct Wide<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

template <int N>
struct Codes;   // N codes in a register or two
template <>
struct Codes<8> {
  using type = uint2;
  static __device__ __forceinline__ uint2 encode(const float (&x)[8], float inv) {
    return make_uint2(e4m3x2(x[0] * inv, x[1] * inv) | (e4m3x2(x[2] * inv, x[3] * inv) << 16),
                      e4m3x2(x[4] * inv, x[5] * inv) | (e4m3x2(x[6] * inv, x[7] * inv) << 16));
  }
  static __device__ __forceinline__ void decode(const uint2& c, float scale, float (&x)[8]) {
    const uint32_t w[4] = {c.x, c.x >> 16, c.y, c.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = e4m3x2_values(w[i]);
      x[2 * i] = v.x * scale, x[2 * i + 1] = v.y * scale;
    }
  }
};
template <>
struct Codes<4> {
  using type = uint32_t;
  static __device__ __forceinline__ uint32_t encode(const float (&x)[4], float inv) {
    return e4m3x2(x[0] * inv, x[1] * inv) | (e4m3x2(x[2] * inv, x[3] * inv) << 16);
  }
  static __device__ __forceinline__ void decode(uint32_t c, float scale, float (&x)[4]) {
    const float2 a = e4m3x2_values(c), b = e4m3x2_values(c >> 16);
    x[0] = a.x * scale, x[1] = a.y * scale, x[2] = b.x * scale, x[3] = b.y * scale;
  }
};

// CTA of kSlots slots, of p.heads heads one after the other. Rows to be written mostly come from a projection, where a
// token's heads are neighbours, so the heads' CTAs of a tile of slots are neighbours too; rows read lie by heads on both
// sides.
enum Kv8 { kRead, kWriteRows, kDecode };

// kDecode: reads, and a row whose K or V is NaN gets a NaN key and a zero value (an attention kernel's weight of
// zero times NaN would be NaN; a NaN score reaches the rows that see the key alone).
template <typename T, int D, Kv8 kKind>
__global__ void __launch_bounds__(kThreads, 6) kv8_kernel(const __grid_constant__ Kv8Params p) {
  constexpr bool kWrite = kKind == kWriteRows;
  using W = Wide<T>;
  constexpr int N = W::kN;
  constexpr int kLanes = D / N;                      // lanes of a row
  constexpr int kSlots = kThreads / kLanes * kTok;   // slots of a CTA
  using C = typename Codes<N>::type;
  __shared__ int s_pos[kSlots];
  griddep_wait();
  griddep_launch_dependents();
  const int tid = threadIdx.x;
  const int b = blockIdx.z;
  const int row = static_cast<int>(blockIdx.y) + p.first;
  const int slot0 = (kWrite ? row : static_cast<int>(blockIdx.x)) * kSlots;
  const int head_group = kWrite ? static_cast<int>(blockIdx.x) : row;
  const int32_t* list = p.pos == nullptr ? nullptr : p.pos + static_cast<size_t>(b) * p.n;
  const int lane = tid % kLanes, group = tid / kLanes;
  // the rows to be written of head h; those of the first are on their way while a list is looked through
  uint4 r[2][kTok];
  const auto load = [&](int h) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const T* x = reinterpret_cast<const T*>(p.src[w]) + b * p.sb[w] + h * p.sh[w] + lane * N;
#pragma unroll
      for (int j = 0; j < kTok; ++j) {
        const int s = slot0 + group * kTok + j;
        r[w][j] = make_uint4(0, 0, 0, 0);
        if (s < p.n) r[w][j] = __ldcs(reinterpret_cast<const uint4*>(x + s * p.sl[w]));
      }
    }
  };
  if (kWrite) load(head_group * p.heads);
  int at[kTok];
  if (list == nullptr) {
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const int s = slot0 + group * kTok + j;
      at[j] = s < p.n ? p.pos0 + s : -1;
    }
  } else {
    for (int i = tid; i < kSlots; i += kThreads) {
      const int s = slot0 + i, x = s < p.n ? __ldg(list + s) : -1;
      s_pos[i] = x >= 0 && x < p.L ? x : -1;
    }
    __syncthreads();
    if (kWrite) {
      // a slot whose position a lower slot names does not write it: a warp looks through the list for kMine slots
      constexpr int kMine = kSlots / (kThreads / 32);
      const int first = (tid >> 5) * kMine;
      int mine[kMine];
#pragma unroll
      for (int k = 0; k < kMine; ++k) mine[k] = s_pos[first + k];
      uint32_t hit = 0;
#pragma unroll 2
      for (int o = tid & 31; o < min(p.n, slot0 + first + kMine); o += 32) {
        const int x = __ldg(list + o);
#pragma unroll
        for (int k = 0; k < kMine; ++k)
          if (x == mine[k] && o < slot0 + first + k) hit |= 1u << k;
      }
      hit = __reduce_or_sync(0xffffffffu, hit);
      if ((tid & 31) < kMine && ((hit >> (tid & 31)) & 1u)) s_pos[first + (tid & 31)] = -1;
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kTok; ++j) at[j] = s_pos[group * kTok + j];
  }
  const int h1 = min(p.Hkv, (head_group + 1) * p.heads);
  for (int h = head_group * p.heads; h < h1; ++h) {
    const size_t mem0 = (static_cast<size_t>(b) * p.Hkv + h) * p.L;   // the head's first memory row
    if (kWrite) {
      if (h > head_group * p.heads) load(h);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
          float x[N];
          W::unpack(r[w][j], x);
          // the largest magnitude by its bits: NaN is above infinity, infinity above every number
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
          for (int o = kLanes / 2; o >= 1; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
          const int e = e4m3_row_exponent(__uint_as_float(top));
          const float inv = e4m3_inverse_scale(e);
          if (e == kExpNan) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.0f;
          }
          const C code = Codes<N>::encode(x, inv);
          if (at[j] >= 0) {
            *reinterpret_cast<C*>(p.dst[w] + (mem0 + at[j]) * D + lane * N) = code;
            if (lane == 0) p.exps[w][mem0 + at[j]] = static_cast<uint8_t>(e);
          }
        }
      }
    } else {
      C c[2][kTok];
      uint8_t e[2][kTok];
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
          c[w][j] = C{};
          e[w][j] = kExpZero;
          if (at[j] >= 0) {
            c[w][j] = __ldcs(reinterpret_cast<const C*>(p.src[w] + (mem0 + at[j]) * D + lane * N));
            e[w][j] = __ldg(p.exps[w] + mem0 + at[j]);
          }
        }
      bool nan[kTok] = {};
      if constexpr (kKind == kDecode) {
        // a row with a NaN code in its K or V counts as a NaN row too
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
          uint32_t hit = 0;
#pragma unroll
          for (int w = 0; w < 2; ++w)
            hit |= ((c[w][j].x & 0x7f7f7f7fu) + 0x01010101u) | ((c[w][j].y & 0x7f7f7f7fu) + 0x01010101u);
          const uint32_t rows = __ballot_sync(0xffffffffu, (hit & 0x80808080u) != 0);
          const uint32_t mine = (0xffffffffu >> (32 - kLanes)) << (tid & 31 & ~(kLanes - 1));
          nan[j] = e[0][j] > kExpMax || e[1][j] > kExpMax || (rows & mine) != 0;
        }
      }
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
          const int s = slot0 + group * kTok + j;
          if (s >= p.n) continue;
          float x[N];
          int byte = e[w][j];
          if (kKind == kDecode) {
            if (nan[j]) c[w][j] = C{}, byte = w ? kExpZero : kExpNan;
          }
          Codes<N>::decode(c[w][j], e4m3_scale(byte), x);
          T* out = reinterpret_cast<T*>(p.dst[w]) + ((static_cast<size_t>(b) * p.Hkv + h) * p.n + s) * D + lane * N;
          *reinterpret_cast<uint4*>(out) = W::pack(x);
        }
    }
  }
}

// Launches the grid's rows, at most 65535 (a grid's height) at a time. (All of a grid in its first
// dimension would leave the kernel an integer division and 28 bytes of spills: 4 x 8 heads of 8191 rows took 50.8 us to
// write instead of 37.9.)
int launch_rows(void (*fn)(const Kv8Params), Kv8Params p, long long columns, long long rows, int B, cudaStream_t stream) {
  for (long long at = 0; at < rows; at += 65535) {
    p.first = static_cast<int>(at);
    cudaLaunchAttribute attr[1];
    const dim3 grid(static_cast<unsigned>(columns), static_cast<unsigned>(std::min<long long>(rows - at, 65535)),
                    static_cast<unsigned>(B));
    const cudaLaunchConfig_t cfg = pdl_config(grid, dim3(kThreads), 0, stream, attr);
    if (cudaLaunchKernelEx(&cfg, fn, p) != cudaSuccess || cudaGetLastError() != cudaSuccess) return -3;
  }
  return 0;
}

template <typename T, int D>
int launch(Kv8Params p, int B, Kv8 kind, cudaStream_t stream) {
  const bool write = kind == kWriteRows;
  constexpr int kSlots = kThreads / (D / Wide<T>::kN) * kTok;
  const long long tiles = (p.n + kSlots - 1) / kSlots;
  if (B > 65535 || p.n > 0x7fffffff - kSlots) return -2;
  // A CTA takes one head; with a list to search for repeats, as many as leave the GPU about two waves
  // of CTAs, so that the search is not made again for each head.
  long long groups = p.Hkv;
  if (write && p.pos != nullptr) groups = std::min<long long>(p.Hkv, std::max<long long>(1, 2 * 152 * 4 / (tiles * B)));
  p.heads = static_cast<int>((p.Hkv + groups - 1) / groups);
  groups = (p.Hkv + p.heads - 1) / p.heads;
  const auto fn = write ? kv8_kernel<T, D, kWriteRows> : kv8_kernel<T, D, kRead>;
  return write ? launch_rows(fn, p, groups, tiles, B, stream) : launch_rows(fn, p, tiles, groups, B, stream);
}

}  // namespace

namespace {

Kv8Params params_of(const Kv8Args& a, bool write) {
  Kv8Params p{};
  for (int w = 0; w < 2; ++w) {
    uint8_t* codes = static_cast<uint8_t*>(w ? a.v8 : a.k8);
    uint8_t* rows = static_cast<uint8_t*>(w ? a.v : a.k);
    p.src[w] = write ? rows : codes;
    p.dst[w] = write ? codes : rows;
    p.exps[w] = w ? a.v_exp : a.k_exp;
    if (write) p.sb[w] = a.strides[3 * w], p.sh[w] = a.strides[3 * w + 1], p.sl[w] = a.strides[3 * w + 2];
  }
  p.pos = a.pos;
  p.pos0 = a.pos0;
  p.n = a.n;
  p.L = a.L;
  p.Hkv = a.Hkv;
  p.heads = 1;
  return p;
}

}  // namespace

int launch_kv8(const Kv8Args& a, bool write, cudaStream_t stream) {
  if (a.n == 0) return 0;
  const Kv8Params p = params_of(a, write);
  const Kv8 kind = write ? kWriteRows : kRead;
  using bf16 = __nv_bfloat16;
  if (a.elem_bytes == 2) return a.D == 64 ? launch<bf16, 64>(p, a.B, kind, stream) : launch<bf16, 128>(p, a.B, kind, stream);
  return a.D == 64 ? launch<float, 64>(p, a.B, kind, stream) : launch<float, 128>(p, a.B, kind, stream);
}

int launch_kv8_decode(const Kv8Args& a, cudaStream_t stream) {
  using bf16 = __nv_bfloat16;
  constexpr int kSlots = kThreads / (128 / Wide<bf16>::kN) * kTok;
  // whole memories lie one behind the other: the heads of all sequences are those of one (a grid's depth is 65535 too)
  Kv8Params p = params_of(a, false);
  const long long heads = static_cast<long long>(a.B) * a.Hkv;
  if (heads > 0x7fffffffLL) return -2;
  p.Hkv = static_cast<int>(heads);
  return launch_rows(kv8_kernel<bf16, 128, kDecode>, p, (a.n + kSlots - 1) / kSlots, heads, 1, stream);
}

}  // namespace cover
