// The 1x1 mix of 8-bit codes (gfx950): out = (codes of a token . codes of a
// weight row) * token scale * weight scale + bias, the product exact in int32.
// Both operands are rows contiguous along the reduction, padded with zeros to
// whole 128 bytes; rows i of one and rows j of the other give out(i, j), with
// the index that is contiguous in the output as j: tokens [T][M] take i =
// token, j = weight row, maps [N][M][P] the reverse.
#include "bc_internal.hpp"
#include "bc_scan.hpp"

namespace bc {
namespace {

using namespace scan;

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

struct Args {
  const int8_t *a, *b;        // rows i, rows j
  const float *ascale, *bscale;
  const float* bias;          // of the weight rows, or null
  char* out;
  int I, J;                   // rows of a and of b
  int pitch, M, P, relu;
};

// out(i, j) of a 32-bit sum.
template <int OUT, bool kMaps>
__device__ __forceinline__ void store_out(const Args& p, int i, int j, int sum, float si, float sj, float bi, float bj) {
  float z = kMaps ? (float)sum * sj * si : (float)sum * si * sj;   // token scale first
  if (p.bias) z += kMaps ? bi : bj;
  if (p.relu) z = z > 0.f || z != z ? z : 0.f;
  const long at = kMaps ? ((long)(j / p.P) * p.M + i) * p.P + j % p.P : (long)i * p.M + j;
  if constexpr (OUT == kBF16) reinterpret_cast<uint16_t*>(p.out)[at] = (uint16_t)pair_bf16(z, 0.f);
  else reinterpret_cast<float*>(p.out)[at] = z;
}

// One wave per 32 x 32 outputs, operands straight from memory.
template <int OUT, bool kMaps>
__global__ __launch_bounds__(256) void k_mix_i8(Args p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nj = (p.J + 63) / 64;
  const int i0 = (int)(blockIdx.x / nj) * 64 + (wave >> 1) * 32, j0 = (int)(blockIdx.x % nj) * 64 + (wave & 1) * 32;
  const int8_t* a = p.a + (long)min(i0 + (lane & 31), p.I - 1) * p.pitch + 16 * (lane >> 5);
  const int8_t* b = p.b + (long)min(j0 + (lane & 31), p.J - 1) * p.pitch + 16 * (lane >> 5);
  i32x16_t acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0;
  for (int k = 0; k < p.pitch; k += 32)
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4_t*>(a + k),
                                                *reinterpret_cast<const i32x4_t*>(b + k), acc, 0, 0, 0);
  const int j = j0 + (lane & 31);
  if (j >= p.J) return;
  const float sj = p.bscale[j], bj = p.bias && !kMaps ? p.bias[j] : 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int i = i0 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
    if (i < p.I) store_out<OUT, kMaps>(p, i, j, acc[r], p.ascale[i], sj, p.bias && kMaps ? p.bias[i] : 0.f, bj);
  }
}

template <int OUT, bool kMaps>
hipError_t launch(const Args& p, hipStream_t s) {
  const dim3 grid((unsigned)(((long)(p.I + 63) / 64) * ((p.J + 63) / 64)));
  hipLaunchKernelGGL((k_mix_i8<OUT, kMaps>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

// Workspace: the tokens' codes, then their scales.
size_t codes_bytes(long rows, int K) { return ((size_t)rows * i8_pitch(K) + 255) & ~(size_t)255; }

}  // namespace

size_t mix_i8_workspace_bytes(int N, int, int K, int P, int dt, bool) {
  if (dt == 3) return 0;   // codes already
  const long rows = (long)N * P;
  return codes_bytes(rows, K) + (size_t)rows * 4;
}

hipError_t launch_mix_i8(const MixI8& m, hipStream_t s) {
  const long rows = (long)m.N * m.P;
  const int8_t* x = static_cast<const int8_t*>(m.x);
  const float* xscale = m.xscale;
  if (m.dt != 3) {
    char* ws = static_cast<char*>(m.ws);
    float* scale = reinterpret_cast<float*>(ws + codes_bytes(rows, m.K));
    const hipError_t e = launch_quantize_i8(m.x, m.dt, m.bs, m.rs, ws, scale, m.N, m.K, m.P, m.maps, s);
    if (e != hipSuccess) return e;
    x = reinterpret_cast<const int8_t*>(ws);
    xscale = scale;
  }
  const int8_t* w = static_cast<const int8_t*>(m.wq);
  Args p{};
  p.bias = m.bias;
  p.out = static_cast<char*>(m.out);
  p.pitch = i8_pitch(m.K);
  p.M = m.M;
  p.P = m.P;
  p.relu = m.relu;
  if (m.maps) {
    p.a = w; p.ascale = m.wscale; p.I = m.M;
    p.b = x; p.bscale = xscale; p.J = (int)rows;
    return m.out_dt == kBF16 ? launch<kBF16, true>(p, s) : launch<kF32, true>(p, s);
  }
  p.a = x; p.ascale = xscale; p.I = (int)rows;
  p.b = w; p.bscale = m.wscale; p.J = m.M;
  return m.out_dt == kBF16 ? launch<kBF16, false>(p, s) : launch<kF32, false>(p, s);
}

}  // namespace bc
