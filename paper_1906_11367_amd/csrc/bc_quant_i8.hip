// 8-bit codes of the rows a mix reduces over (gfx950): for K values x of one
// token (or of one weight row), with m = max |x|,
//   scale = m / 127,  q = round to nearest even(x * (127 / m)),
// in fp32, all zero where m < 2^-100 (127 / m would leave fp32's range); a row
// with a NaN or an infinity gets a NaN scale, so that every output made from
// it is NaN.  Rows of codes are padded with zeros to whole 128 bytes, which
// leaves the products no tail along the reduction.
// Bound by memory: one read of x (the second comes from cache) and a byte out
// for each value.
#include "bc_internal.hpp"
#include "bc_scan.hpp"   // load_vec, elem

namespace bc {
namespace {

using namespace scan;

constexpr uint32_t kInfBits = 0x7f800000u;

struct RowScale { float inv, scale; };

// top: the largest |x| of the row as bits (a NaN's are above infinity's).
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  const float m = __uint_as_float(top);
  if (top >= kInfBits) return {0.f, __uint_as_float(0x7fc00000u)};
  if (m < 0x1p-100f) return {0.f, 0.f};
  return {127.f / m, m / 127.f};
}

// inv = 0: a row of zeros whatever it holds (NaN * 0 converts to 0).
__device__ __forceinline__ uint32_t code(float v, float inv) {
  return (uint32_t)(int)rintf(inv == 0.f ? 0.f : v * inv) & 0xffu;
}

template <int V>
__device__ __forceinline__ uint32_t top_bits(uint32_t top, const float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
  return top;
}

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
    float v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = elem<DT, 16>(r, k);
    top = top_bits(top, v);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const RowScale s = row_scale(top);
  for (int k0 = lane * 16; k0 < pitch; k0 += 1024) {
    const auto r = load_vec<DT, 16>(p + (long)k0 * kBytes<DT>, K - k0);
    Raw<4> out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      out[w] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) out[w] |= code(elem<DT, 16>(r, 4 * w + k), s.inv) << (8 * k);
    }
    *reinterpret_cast<Raw<4>*>(q + row * pitch + k0) = out;
  }
  if (lane == 0) scale[row] = s.scale;
}

// Maps [N][K][P] to rows of tokens: a block takes 64 pixels of one image, a
// lane one pixel; its four waves share the channels.
template <int DT>
__global__ __launch_bounds__(256) void k_quant_maps(const char* src, long bs, long rs, int8_t* q, float* scale, int P,
                                                    int K, int pitch, int strips) {
  __shared__ uint32_t tops[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = blockIdx.x / strips, p = (blockIdx.x % strips) * 64 + lane;
  const bool on = p < P;
  const char* base = src + ((long)n * bs + p) * kBytes<DT>;
  auto at = [&](int k) { return elem<DT, 2>(load_vec<DT, 2>(base + (long)k * rs * kBytes<DT>, on && k < K ? 1 : 0), 0); };
  uint32_t top = 0;
  for (int k = wave; k < K; k += 4) top = max(top, __float_as_uint(at(k)) & 0x7fffffffu);
  tops[wave][lane] = top;
  __syncthreads();
  top = max(max(tops[0][lane], tops[1][lane]), max(tops[2][lane], tops[3][lane]));
  const RowScale s = row_scale(top);
  const long row = (long)n * P + p;
  for (int k0 = wave * 16; k0 < pitch; k0 += 64) {
    Raw<4> out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      out[w] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) out[w] |= code(at(k0 + 4 * w + k), s.inv) << (8 * k);
    }
    if (on) *reinterpret_cast<Raw<4>*>(q + row * pitch + k0) = out;
  }
  if (on && wave == 0) scale[row] = s.scale;
}

}  // namespace

hipError_t launch_quantize_i8(const void* src, int dt, long bs, long rs, void* q, float* scale, int N, int K, int P,
                              bool maps, hipStream_t s) {
  const char* x = static_cast<const char*>(src);
  int8_t* out = static_cast<int8_t*>(q);
  const int pitch = i8_pitch(K);
  if (maps) {
    const int strips = (P + 63) / 64;
    const dim3 grid((unsigned)((long)N * strips));
    if (dt == kBF16) hipLaunchKernelGGL((k_quant_maps<kBF16>), grid, dim3(256), 0, s, x, bs, rs, out, scale, P, K, pitch, strips);
    else hipLaunchKernelGGL((k_quant_maps<kF32>), grid, dim3(256), 0, s, x, bs, rs, out, scale, P, K, pitch, strips);
  } else {
    const long rows = (long)N * P;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (dt == kBF16) hipLaunchKernelGGL((k_quant_rows<kBF16>), grid, dim3(256), 0, s, x, bs, rs, out, scale, rows, P, K, pitch);
    else hipLaunchKernelGGL((k_quant_rows<kF32>), grid, dim3(256), 0, s, x, bs, rs, out, scale, rows, P, K, pitch);
  }
  return hipGetLastError();
}

}  // namespace bc
