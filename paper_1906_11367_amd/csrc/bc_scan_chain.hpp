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

}  // namespace scan
}  // namespace bc
