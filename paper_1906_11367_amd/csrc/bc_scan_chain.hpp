// How the blocks of a chained scan share the work (bc_scan.hip), as functions of
// numbers alone: they run on the host too.
#pragma once
#include <hip/hip_runtime.h>

namespace bc {
namespace scan {

// The unit (a slab of a sequence) of block b < units * tiles; every unit has
// `tiles` blocks.  Blocks go to the XCDs in turn: neighbouring units to one XCD.
__host__ __device__ inline int chain_unit(long b, int units) {
  const int u = (int)(b % units), eighth = units >> 3;
  return u < eighth * 8 ? (u & 7) * eighth + (u >> 3) : u;
}

// A drawn number is a place of the chain.  The counter, which starts at -1, gives
// a call of its own workspace the numbers 0 .. tiles - 1; where another call
// writes the same workspace meanwhile it may give any, and the tile of one
// outside would lie outside the tensors.
__host__ __device__ inline bool chain_has(int place, int tiles) { return (unsigned)place < (unsigned)tiles; }

// The rows and columns of a grid of `blocks` or a few more (those return): a grid
// has less than 2^32 threads along x, and blocks have 512 at most.
struct Grid { unsigned x, y; };
inline Grid grid_of(long blocks) {
  const long x = blocks < 1L << 22 ? blocks : 1L << 22;
  return {(unsigned)x, (unsigned)((blocks + x - 1) / x)};
}

// Blocks that fill a call's words, two to a thread of 256.
inline long clear_blocks(long words) { return (words + 511) / 512; }

}  // namespace scan
}  // namespace bc
