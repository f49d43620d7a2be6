// 8-bit codes and scales of the rows a mix reduces over (gfx950; bc_i8.hpp has
// the definition).  Rows of codes are padded with zeros to whole 128 bytes,
// which leaves the products no tail along the reduction.
// Bound by memory: one read of x and a byte out for each value.  16384 rows of 4096
// bf16: 33 us (201 MB at 6.1 TB/s, part of it from the last-level cache); 8 images
// of 1024 x 64 x 64 bf16 34 to 41, of 3000 108: channels that registers do not hold
// until a pixel's scale is known (past 1024 in bf16, 512 in fp32) are read again,
// counted 357 MB for 197, and 131 written for 101; the 488 MB pass at 4.5 TB/s.
#include "bc_i8.hpp"

#include <algorithm>

namespace bc {
namespace {

using namespace i8;

// Rows of tokens: W waves to a row, 16 values a lane at a time.  The first two
// pieces of a row (2048 W values) stay in registers; the rest is read again.
constexpr int kHeldPieces = 2;

template <int DT, int W>
__global__ __launch_bounds__(256) void k_quant_rows(const char* src, long bs, long rs, int8_t* q, float* scale,
                                                    long rows, int P, int K, int pitch) {
  constexpr int kPiece = W * 1024;
  __shared__ uint32_t tops[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k1 = (threadIdx.x & (64 * W - 1)) * 16;
  const long b = (long)blockIdx.y * gridDim.x + blockIdx.x, row = W == 4 ? b : b * 4 + wave;
  if (row >= rows) return;   // W = 4: the whole block
  const char* p = src + ((row / P) * bs + (row % P) * rs) * kBytes<DT>;
  auto load = [&](int k) { return load_vec<DT, 16>(p + (long)k * kBytes<DT>, K - k); };
  Raw<kWords<DT, 16>> x[kHeldPieces];
  if (K >= kHeldPieces * kPiece) {   // all there, for every lane
#pragma unroll
    for (int i = 0; i < kHeldPieces; ++i) x[i] = load_wide<DT, 16>(p + (long)(k1 + i * kPiece) * kBytes<DT>);
  } else if (K == kPiece) {
    x[0] = load_wide<DT, 16>(p + (long)k1 * kBytes<DT>);
    x[1] = Raw<kWords<DT, 16>>{};
  } else {
#pragma unroll
    for (int i = 0; i < kHeldPieces; ++i) x[i] = load(k1 + i * kPiece);
  }
  Largest<DT, 16> largest;
#pragma unroll
  for (int i = 0; i < kHeldPieces; ++i) largest.take(x[i]);
  for (int k = k1 + kHeldPieces * kPiece; k < K; k += kPiece) largest.take(load(k));
  uint32_t top = largest.all();
#pragma unroll
  for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if constexpr (W == 4) {
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  const RowScale s = row_scale(top);
  auto put = [&](int k, const Raw<kWords<DT, 16>>& r) {
    if (k >= pitch) return;
    Raw<4> out;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      out[w] = codes4(elem<DT, 16>(r, 4 * w), elem<DT, 16>(r, 4 * w + 1), elem<DT, 16>(r, 4 * w + 2),
                      elem<DT, 16>(r, 4 * w + 3), s.inv);
    *reinterpret_cast<Raw<4>*>(q + row * pitch + k) = out;
  };
#pragma unroll
  for (int i = 0; i < kHeldPieces; ++i) put(k1 + i * kPiece, x[i]);
  for (int k = k1 + kHeldPieces * kPiece; k < pitch; k += kPiece) put(k, load(k));
  if (k1 == 0) scale[row] = s.scale;
}

// Maps [N][K][P] to rows of tokens: a block takes PX pixels of one image, and
// turns them through LDS, up to kPart steps of channels at a time.
template <int PX> constexpr int kPart = PX == 64 ? 4 : 2;

template <int DT, int PX, int kHold, bool kFull>
__device__ __forceinline__ void quant_tile(const char* base, long rs, const Pixels& at, int8_t* q, int left, int K, int pitch,
                                           int steps, uint32_t lds, uint32_t* tops, RowScale* rows) {
  constexpr int Step = kStepK<PX>;
  const int tid = threadIdx.x, lp = min(steps, kPart<PX>) * Step;
  Raw<kWords<DT, 8>> x[kHold + 1][4];
  tile_scales<DT, PX, kHold, kFull>(base, rs, at, K, x, tops, rows);
  for (int s0 = 0; s0 < steps; s0 += kPart<PX>) {
    const int s1 = min(steps, s0 + kPart<PX>);
    if (s0 > 0) __syncthreads();
    tile_codes<DT, PX, kHold, kFull>(base, rs, at, K, x, rows, lds, lp, s0, s1);
    __syncthreads();
    // whole rows out, 16 bytes a lane
    const int chunks = min(pitch - s0 * Step, (s1 - s0) * Step) >> 4;
    for (int c = tid; c < PX * chunks; c += kTileThreads) {
      const int p = c / chunks, ch = c % chunks;
      if (p >= left) break;
      const Raw<4> w = *(BC_LDS Raw<4>*)(uintptr_t)(lds + p * lp + ((ch ^ chunk_swap<PX>(p)) << 4));
      *reinterpret_cast<Raw<4>*>(q + (long)p * pitch + s0 * Step + ch * 16) = w;
    }
  }
}

template <int DT, int PX>
__global__ __launch_bounds__(kTileThreads, 4) void k_quant_maps(const char* src, long bs, long rs, int8_t* q,
                                                                float* scale, int P, int K, int pitch, int strips,
                                                                int steps, bool near) {
  extern __shared__ __align__(16) unsigned char smem[];   // codes of the pixels
  __shared__ uint32_t tops[kTileThreads / 64 * PX];
  __shared__ RowScale rows[PX];
  const int b = tile_of_block(near), tid = threadIdx.x, n = b / strips, pt = (b % strips) * PX, left = P - pt;
  const Pixels at(tid % (PX / 8) * 8, left, P);
  const uint32_t lds = (uint32_t)(uintptr_t)(BC_LDS unsigned char*)smem;
  const char* base = src + ((long)n * bs + pt + at.first) * kBytes<DT>;
  int8_t* out = q + ((long)n * P + pt) * pitch;
  if (left >= PX) quant_tile<DT, PX, kHeld<DT>, true>(base, rs, at, out, left, K, pitch, steps, lds, tops, rows);
  else quant_tile<DT, PX, kHeld<DT>, false>(base, rs, at, out, left, K, pitch, steps, lds, tops, rows);
  if (tid < PX && tid < left) scale[(long)n * P + pt + tid] = rows[tid].scale;
}

template <int DT, int PX>
hipError_t launch_maps(const char* x, long bs, long rs, int8_t* q, float* scale, int N, int P, int K, int pitch,
                       hipStream_t s) {
  const int strips = (P + PX - 1) / PX, steps = (pitch + kStepK<PX> - 1) / kStepK<PX>;
  const size_t lds = (size_t)PX * std::min(steps, kPart<PX>) * kStepK<PX>;
  // rows, or a strip's part of one, that are not whole 64 bytes (4096 x 64 x 64
  // bf16, strips of 16: 16 us with neighbours, 28 in order; 2 x 957 x 1072 fp32,
  // whole 64 bytes, 12 and 11)
  const bool near = rs % (64 / kBytes<DT>) != 0 || PX * kBytes<DT> % 64 != 0;
  hipLaunchKernelGGL((k_quant_maps<DT, PX>), dim3((unsigned)((long)N * strips)), dim3(kTileThreads), lds, s, x, bs, rs,
                     q, scale, P, K, pitch, strips, steps, near);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_i8(const void* src, int dt, long bs, long rs, void* q, float* scale, int N, int K, int P,
                              bool maps, hipStream_t s) {
  const char* x = static_cast<const char*>(src);
  int8_t* out = static_cast<int8_t*>(q);
  const int pitch = i8_pitch(K);
  if (maps) {
    // narrow strips where wide ones leave the chip empty
    const bool narrow = (long)N * ((P + 63) / 64) < 256;
    if (dt == kBF16)
      return narrow ? launch_maps<kBF16, 16>(x, bs, rs, out, scale, N, P, K, pitch, s)
                    : launch_maps<kBF16, 64>(x, bs, rs, out, scale, N, P, K, pitch, s);
    return narrow ? launch_maps<kF32, 16>(x, bs, rs, out, scale, N, P, K, pitch, s)
                  : launch_maps<kF32, 64>(x, bs, rs, out, scale, N, P, K, pitch, s);
  } else {
    const long rows = (long)N * P;
    const bool block = K > 2 * 1024 || rows < 1024;   // a block to a row
    const long blocks = block ? rows : (rows + 3) / 4, across = std::min(blocks, 1L << 22);
    const dim3 grid((unsigned)across, (unsigned)((blocks + across - 1) / across));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, x, bs, rs, out, scale, rows, P, K, pitch); };
    if (dt == kBF16) block ? go(k_quant_rows<kBF16, 4>) : go(k_quant_rows<kBF16, 1>);
    else block ? go(k_quant_rows<kF32, 4>) : go(k_quant_rows<kF32, 1>);
  }
  return hipGetLastError();
}

}  // namespace bc
