// paged_ring.cuh - the order of the few-rows kernel's copies over a memory in pages (attn_paged.cu), the places that they take in shared
// memory and the barriers that they complete.
//
// A wait tells a phase of its barrier from the one before it by a parity alone, so the phase behind the one that is waited for must not
// complete before the wait has passed, and the one before it must have completed by then. Places do not give barriers of that kind: K's
// place is free as soon as its scores are there, whether or not the warps that look V through have got that far, and the copy that takes it could
// complete a second phase before they look at the first. So a tile's K and V have barriers of their own, each in turns of kBarriers tiles: the warps
// wait for V's alone, and V of tile g + 3, whose place K of g + 2 had (or, last of all, V of g), is not asked for before the products with V of g, nor
// those before V of g has been looked through.
#pragma once

#ifdef __CUDACC__
#define COVER_RING_FN __host__ __device__ constexpr
#else
#define COVER_RING_FN constexpr
#endif

namespace cover {
namespace paged_ring {

constexpr int kSlots = 5;      // tiles of K or V in shared memory, taken in turn
constexpr int kBarriers = 4;   // of K and of V

struct Copy {
  bool is_v;
  int tile;
};

// The i-th of the 2 n copies of n tiles: K0, K1, V0, K2, V1, .., K(n-1), V(n-2), V(n-1).
COVER_RING_FN Copy copy_at(int i, int n) {
  const bool last = i == 2 * n - 1, is_v = last || (i > 0 && (i & 1) == 0);
  return Copy{is_v, last ? n - 1 : is_v ? i / 2 - 1 : (i + 1) / 2};
}
COVER_RING_FN int copy_of_k(int tile) { return tile == 0 ? 0 : 2 * tile - 1; }
COVER_RING_FN int copy_of_v(int tile, int n) { return tile == n - 1 ? 2 * n - 1 : 2 * tile + 2; }
COVER_RING_FN int slot_of(int copy) { return copy % kSlots; }
COVER_RING_FN int barrier_of(int tile) { return tile % kBarriers; }
COVER_RING_FN int phase_of(int tile) { return tile / kBarriers; }

}  // namespace paged_ring
}  // namespace cover
