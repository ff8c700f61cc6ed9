// tmap.cuh - host-side creation of TMA tensor maps through the driver entry
// point (no link-time dependency on libcuda).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cover {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Returns nullptr if the driver does not provide cuTensorMapEncodeTiled.
EncodeTiledFn encode_tiled_fn();

// bf16 tensor viewed as 4-D (d0 fastest) with 128-byte swizzle and a box of
// {64, box1, 1, 1} elements; out-of-range elements read as zero.
bool make_bf16_map_4d(CUtensorMap* map, const void* base, uint64_t d0, uint64_t d1, uint64_t d2, uint64_t d3,
                      uint32_t box1);

// The same for bytes: a 4-D tensor [d3][d2][d1][d0] of uint8, a box of box1 rows of 128 columns, 128-byte swizzle.
bool make_u8_map_4d(CUtensorMap* map, const void* base, uint64_t d0, uint64_t d1, uint64_t d2, uint64_t d3, uint32_t box1);

// Rows of 128 bf16 (16-byte aligned, 256 bytes apart) as groups of eight, and boxes of box_groups of them: in shared memory a group is its rows' first
// 64 columns (8 x 128 bytes, 128-byte swizzle), then their last 64. Coordinates {0, 0, 0, group}; groups outside read as zero.
bool make_bf16_row_groups_map(CUtensorMap* map, const void* base, uint64_t groups, uint32_t box_groups);

}  // namespace cover
