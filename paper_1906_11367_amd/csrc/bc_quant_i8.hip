// 8-bit codes and scales of the rows a mix reduces over (gfx950; bc_i8.hpp has
// the definition).  Rows of codes are padded with zeros to whole 128 bytes,
// which leaves the products no tail along the reduction.
// Bound by memory: one read of x and a byte out for each value.
#include "bc_i8.hpp"

#include <algorithm>

namespace bc {
namespace {

using namespace i8;

// Rows of tokens: a wave per row, 16 values a lane at a time.
template <int DT>
__global__ __launch_bounds__(256) void k_quant_rows(const char* src, long bs, long rs, int8_t* q, float* scale,
                                                    long rows, int P, int K, int pitch) {
  const int lane = threadIdx.x & 63;
  const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const char* p = src + ((row / P) * bs + (row % P) * rs) * kBytes<DT>;
  uint32_t top = 0;
  for (int k0 = lane * 16; k0 < K; k0 += 1024) {
    const auto r = load_vec<DT, 16>(p + (long)k0 * kBytes<DT>, K - k0);
#pragma unroll
    for (int k = 0; k < 16; ++k) top = max(top, abs_bits(elem<DT, 16>(r, k)));
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const RowScale s = row_scale(top);
  for (int k0 = lane * 16; k0 < pitch; k0 += 1024) {
    const auto r = load_vec<DT, 16>(p + (long)k0 * kBytes<DT>, K - k0);
    Raw<4> out;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      out[w] = codes4(elem<DT, 16>(r, 4 * w), elem<DT, 16>(r, 4 * w + 1), elem<DT, 16>(r, 4 * w + 2),
                      elem<DT, 16>(r, 4 * w + 3), s.inv);
    *reinterpret_cast<Raw<4>*>(q + row * pitch + k0) = out;
  }
  if (lane == 0) scale[row] = s.scale;
}

// Maps [N][K][P] to rows of tokens: a block takes 64 pixels of one image, and
// turns them through LDS, up to kPart steps of 256 channels at a time.
constexpr int kPart = 4;

template <int DT, int kHold, bool kFull>
__device__ __forceinline__ void quant_tile(const char* base, long rs, int avail, int8_t* q, int left, int K, int pitch,
                                           int steps, uint32_t lds, uint32_t* tops, RowScale* rows) {
  const int tid = threadIdx.x, lp = min(steps, kPart) * kStepK;
  Raw<kWords<DT, 8>> x[kHold + 1][4];
  tile_scales<DT, kHold, kFull>(base, rs, avail, K, x, tops, rows);
  for (int s0 = 0; s0 < steps; s0 += kPart) {
    const int s1 = min(steps, s0 + kPart);
    if (s0 > 0) __syncthreads();
    tile_codes<DT, kHold, kFull>(base, rs, avail, K, x, rows, lds, lp, s0, s1);
    __syncthreads();
    // whole rows out, 16 bytes a lane
    const int chunks = min(pitch - s0 * kStepK, (s1 - s0) * kStepK) >> 4;
    for (int c = tid; c < kTileP * chunks; c += kTileThreads) {
      const int p = c / chunks, ch = c % chunks;
      if (p >= left) break;
      const Raw<4> w = *(BC_LDS Raw<4>*)(uintptr_t)(lds + p * lp + ((ch ^ chunk_swap(p)) << 4));
      *reinterpret_cast<Raw<4>*>(q + (long)p * pitch + s0 * kStepK + ch * 16) = w;
    }
  }
}

template <int DT>
__global__ __launch_bounds__(kTileThreads, 4) void k_quant_maps(const char* src, long bs, long rs, int8_t* q,
                                                                float* scale, int P, int K, int pitch, int strips,
                                                                int steps) {
  extern __shared__ __align__(16) unsigned char smem[];   // codes of 64 pixels
  __shared__ uint32_t tops[kTileThreads / 64 * kTileP];
  __shared__ RowScale rows[kTileP];
  const int tid = threadIdx.x, n = blockIdx.x / strips, pt = (blockIdx.x % strips) * kTileP, left = P - pt;
  const int p0 = pt + (tid & 7) * 8;
  const uint32_t lds = (uint32_t)(uintptr_t)(BC_LDS unsigned char*)smem;
  const char* base = src + ((long)n * bs + p0) * kBytes<DT>;
  int8_t* out = q + ((long)n * P + pt) * pitch;
  if (left >= kTileP) quant_tile<DT, kHeld<DT>, true>(base, rs, P - p0, out, left, K, pitch, steps, lds, tops, rows);
  else quant_tile<DT, kHeld<DT>, false>(base, rs, P - p0, out, left, K, pitch, steps, lds, tops, rows);
  if (tid < kTileP && tid < left) scale[(long)n * P + pt + tid] = rows[tid].scale;
}

}  // namespace

hipError_t launch_quantize_i8(const void* src, int dt, long bs, long rs, void* q, float* scale, int N, int K, int P,
                              bool maps, hipStream_t s) {
  const char* x = static_cast<const char*>(src);
  int8_t* out = static_cast<int8_t*>(q);
  const int pitch = i8_pitch(K);
  if (maps) {
    const int strips = (P + kTileP - 1) / kTileP, steps = (pitch + kStepK - 1) / kStepK;
    const dim3 grid((unsigned)((long)N * strips));
    const size_t lds = (size_t)kTileP * std::min(steps, kPart) * kStepK;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), lds, s, x, bs, rs, out, scale, P, K, pitch, strips, steps);
    };
    dt == kBF16 ? go(k_quant_maps<kBF16>) : go(k_quant_maps<kF32>);
  } else {
    const long rows = (long)N * P;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (dt == kBF16) hipLaunchKernelGGL((k_quant_rows<kBF16>), grid, dim3(256), 0, s, x, bs, rs, out, scale, rows, P, K, pitch);
    else hipLaunchKernelGGL((k_quant_rows<kF32>), grid, dim3(256), 0, s, x, bs, rs, out, scale, rows, P, K, pitch);
  }
  return hipGetLastError();
}

}  // namespace bc
