// Shared device code of the 8-bit codes (gfx950): for K values x of one token
// (or of one weight row), with m = max |x|,
//   scale = m / 127,  q = round to nearest even(x * (127 / m)),
// in fp32, all zero where m < 2^-100 (127 / m would leave fp32's range); a row
// with a NaN or an infinity gets zero codes and a NaN scale, so that every
// output made from it is NaN.
#pragma once
#include "bc_internal.hpp"
#include "bc_scan.hpp"   // load_vec, elem

namespace bc {
namespace i8 {

using namespace scan;

#define BC_LDS __attribute__((address_space(3)))

struct RowScale { float inv, scale; };

// top: the largest |x| of the row as bits (a NaN's are above infinity's).
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  const float m = __uint_as_float(top);
  if (top >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u)};
  if (m < 0x1p-100f) return {0.f, 0.f};
  return {127.f / m, m / 127.f};
}

// The largest |x| of elements that stand in one place of several vectors, as
// bits: bf16 two at a time, as they are stored.
template <int DT, int V>
struct Largest {
  Raw<kWords<DT, V>> m = {};
  __device__ __forceinline__ void take(const Raw<kWords<DT, V>>& x) {
    typedef unsigned short U16 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int w = 0; w < kWords<DT, V>; ++w) {
      const uint32_t a = m[w], b = x[w];   // words of their own: a bit cast of a vector's element takes the vector's first
      if constexpr (DT == kBF16)
        m[w] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(U16, a),
                                                                      __builtin_bit_cast(U16, b & 0x7fff7fffu)));
      else
        m[w] = max(a, b & 0x7fffffffu);
    }
  }
  // of element k; of all of them
  __device__ __forceinline__ uint32_t at(int k) const { return __float_as_uint(elem<DT, V>(m, k)); }
  __device__ __forceinline__ uint32_t all() const {
    uint32_t t = 0;
#pragma unroll
    for (int k = 0; k < V; ++k) t = max(t, at(k));
    return t;
  }
};

// Four codes in a word.  Adding 1.5 * 2^23 to the rounded product rounds it to
// the nearest even integer and leaves that in the low byte; inv = 0 (a row
// without codes, whatever it holds) gives zeros.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
#pragma clang fp contract(off)   // the product is rounded before the sum
  constexpr float kMagic = 12582912.f;
  const uint32_t qa = __float_as_uint(a * inv + kMagic), qb = __float_as_uint(b * inv + kMagic);
  const uint32_t qc = __float_as_uint(c * inv + kMagic), qd = __float_as_uint(d * inv + kMagic);
  const uint32_t lo = __builtin_amdgcn_perm(qb, qa, 0x0c0c0400u), hi = __builtin_amdgcn_perm(qd, qc, 0x04000c0cu);
  return inv == 0.f ? 0u : lo | hi;
}

// A tile of maps [K][P]: PX pixels (64, 32 or 16) by all K channels, by a block
// of 512 threads.  A lane has 8 pixels (pg = tid % (PX / 8)) of 4 consecutive
// channels (group kg = tid / (PX / 8)) at a time, kStepK channels in the block:
// loads are runs of PX pixels, and four codes of a pixel make a word.
constexpr int kTileThreads = 512;
template <int PX> constexpr int kStepK = kTileThreads / (PX / 8) * 4;

// The codes of pixel p stand in LDS as a row of whole steps (a multiple of 256
// bytes), its 16-byte chunk c at c ^ chunk_swap(p).  The reads of one chunk of
// 16 consecutive pixels, and the words that a wave writes (a pixel in 8, and
// 16 * 8 / PX consecutive chunks), then hit all banks.
template <int PX>
__device__ __forceinline__ int chunk_swap(int p) {
  if constexpr (PX == 64) return (((p ^ (p >> 3)) & 7) << 1) | ((p >> 3) & 1);
  else if constexpr (PX == 32) return ((p >> 1) & 3) | (((p ^ (p >> 4)) & 1) << 2) | (p & 8);
  else return p & 15;
}

// The tile of this block.  Blocks go to the XCDs in turn; near: neighbouring tiles
// to one XCD, where they share cache lines.
__device__ __forceinline__ int tile_of_block(bool near) {
  const int b = blockIdx.x, eighth = gridDim.x >> 3;
  return near && b < eighth * 8 ? (b & 7) * eighth + (b >> 3) : b;
}

// The 8 pixels of a lane, from the tile's pixel `first` on.  In a row's last tile
// the lanes that pass its end take the 8 before the end again (the same values in
// the same places; pixels before the tile are left out), so that every load is a
// wide one; a row of less than 8 pixels is read piece by piece (short).
struct Pixels {
  int first, avail;
  bool short_row;
  __device__ __forceinline__ Pixels(int lane_first, int left, int P)
      : first(P < 8 ? lane_first : min(lane_first, left - 8)), avail(left - first), short_row(P < 8) {}
};

// The lane's 8 pixels of channel k.  kFull: a tile of whole rows.
template <int DT, bool kFull>
__device__ __forceinline__ Raw<kWords<DT, 8>> tile_load(const char* base, long rs, const Pixels& at, int k, int K) {
  const char* p = base + (long)k * rs * kBytes<DT>;
  if (kFull || !at.short_row) {   // for all lanes of the block
    Raw<kWords<DT, 8>> r = {};
    if (k < K) r = __builtin_bit_cast(Raw<kWords<DT, 8>>, *reinterpret_cast<const Loose<kWords<DT, 8>, kBytes<DT>>*>(p));
    return r;
  } else {
    return load_vec<DT, 8>(p, k < K ? at.avail : 0);
  }
}

// Row scales of the tile.  base: the lane's pixels at channel 0, rs elements
// between channels.  The first kHold steps of channels stay in registers (x);
// later ones are read again for their codes.
// tops: 8 x PX words of LDS, rows: PX RowScales of LDS, whole after the call.
template <int DT, int PX, int kHold, bool kFull>
__device__ __forceinline__ void tile_scales(const char* base, long rs, const Pixels& at, int K,
                                            Raw<kWords<DT, 8>> (&x)[kHold + 1][4], uint32_t* tops, RowScale* rows) {
  constexpr int PL = PX / 8, Step = kStepK<PX>;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kg = tid / PL;
#pragma unroll
  for (int s = 0; s < kHold; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[s][i] = tile_load<DT, kFull>(base, rs, at, s * Step + kg * 4 + i, K);
  Largest<DT, 8> largest;
#pragma unroll
  for (int s = 0; s < kHold; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) largest.take(x[s][i]);
  for (int s = kHold; s * Step < K; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[kHold][i] = tile_load<DT, kFull>(base, rs, at, s * Step + kg * 4 + i, K);
#pragma unroll
    for (int i = 0; i < 4; ++i) largest.take(x[kHold][i]);
  }
  uint32_t top[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) top[j] = largest.at(j);
#pragma unroll
  for (int d = PL; d < 64; d *= 2)
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], d));
  if (lane < PL) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (kFull || at.first + j >= 0) tops[wave * PX + at.first + j] = top[j];
  }
  __syncthreads();
  if (tid < PX) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kTileThreads / 64; ++w) m = max(m, tops[w * PX + tid]);
    rows[tid] = row_scale(m);
  }
  __syncthreads();
}

// Codes of the channels of steps [s0, s1) into LDS at `lds`, for the rows scaled
// above.
template <int DT, int PX, int kHold, bool kFull>
__device__ __forceinline__ void tile_codes(const char* base, long rs, const Pixels& at, int K,
                                           Raw<kWords<DT, 8>> (&x)[kHold + 1][4], const RowScale* rows, uint32_t lds,
                                           int pitch, int s0, int s1) {
  constexpr int PL = PX / 8, Step = kStepK<PX>;
  const int kg = threadIdx.x / PL, p0 = at.first;
  float inv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) inv[j] = rows[kFull ? p0 + j : max(p0 + j, 0)].inv;
  auto put = [&](int s, const Raw<kWords<DT, 8>> (&y)[4]) {
    const int k = (s - s0) * Step + kg * 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t w = codes4(elem<DT, 8>(y[0], j), elem<DT, 8>(y[1], j), elem<DT, 8>(y[2], j), elem<DT, 8>(y[3], j), inv[j]);
      const int p = p0 + j;
      if (kFull || p >= 0) *(BC_LDS uint32_t*)(uintptr_t)(lds + p * pitch + (((k >> 4) ^ chunk_swap<PX>(p)) << 4) + (k & 15)) = w;
    }
  };
  // the words stay as loaded: unpacked values are not kept from the scales on
#pragma unroll
  for (int s = 0; s < kHold; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("" : "+v"(x[s][i]));
#pragma unroll
  for (int s = 0; s < kHold; ++s)
    if (s >= s0 && s < s1) put(s, x[s]);
  for (int s = max(s0, kHold); s < s1; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[kHold][i] = tile_load<DT, kFull>(base, rs, at, s * Step + kg * 4 + i, K);
    put(s, x[kHold]);
  }
}

// Steps held in registers: 16 words of x a step in bf16, 32 in fp32.
template <int DT> constexpr int kHeld = DT == kBF16 ? 4 : 2;

}  // namespace i8
}  // namespace bc
