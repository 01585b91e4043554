// What the tile kernels of both product families share: launch order, exchanges between lane groups, the offset of what is not there.
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

constexpr uint32_t kAbsent = 0x80000000u;   // offset beyond every extent the host lets through

// What lanes 32 .. 63 of a hold for what lanes 0 .. 31 of b hold; odd rows of 16 lanes of a for even rows of b
__device__ __forceinline__ void swap32(unsigned& a, unsigned& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0]; b = r[1];
}
__device__ __forceinline__ void swap16(unsigned& a, unsigned& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0]; b = r[1];
}

// Launch order -> tile: each XCD (own L2; blocks are dealt to the XCDs round-robin) works through a contiguous
// range of tiles, and inside a batch item consecutive tiles walk groups of tile_group tile rows column by column,
// so that the blocks an XCD runs at one time share operand tiles of both kinds in its L2.
struct tile_id { int bx, by, bz; };
__device__ __forceinline__ tile_id tile_of_index(unsigned t, unsigned gx, unsigned gy, unsigned total, int tile_group) {
  {   // XCD x = launch index mod 8 takes the x-th of eight contiguous ranges (the first total mod 8 ranges one tile longer)
    const unsigned x = t & 7u, rem = total & 7u;
    t = x * (total >> 3) + (x < rem ? x : rem) + (t >> 3);
  }
  tile_id id;
  const unsigned per = gx * gy;
  id.bz = t / per;
  const unsigned r = t - id.bz * per;
  const unsigned gm = tile_group > 1 ? (unsigned)tile_group : 1u;
  const unsigned gsz = gm * gx;
  const unsigned grp = r / gsz, first = grp * gm;
  const unsigned rows = gy - first < gm ? gy - first : gm;
  const unsigned q = r - grp * gsz;
  id.by = first + q % rows;
  id.bx = q / rows;
  return id;
}
// Consecutive tiles walk groups of this many tile rows, by the number of tile columns
inline int tile_group_of(unsigned columns) { return columns >= 64 ? 4 : columns >= 12 ? 2 : 1; }
