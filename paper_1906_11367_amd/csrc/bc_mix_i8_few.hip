// The 1x1 mix in 8-bit codes for few tokens (gfx950): a decoding batch.
//
// Bound by the weights, which are read once: M K bytes, and too little
// arithmetic to matter.  A block takes 16 weight rows; its waves share the
// reduction, 128 codes at a time in turn, so that every wave has all of its
// loads in flight at once, and add their int32 sums through LDS (exact, so in
// any order).  A few tokens' codes are made in the block itself, while its
// weights are on the way; more tokens' come from quantize_i8's kernel, and where
// the weight rows leave CUs idle, blocks divide the tokens too.
// 1 token 4096 -> 8192: 9 to 10 us (33.6 MB at 3.5 TB/s); 24 tokens 2048 -> 8192: 6.8.
#include "bc_i8.hpp"

#include <math.h>

namespace bc {
namespace {

using namespace i8;

typedef int i32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kAhead = 4;      // blocks of 128 codes a wave loads together
constexpr int kItems = 4;      // pieces of 512 values a wave turns into codes

struct Args {
  const int8_t* w;
  const float *wscale, *bias;
  const char* x;               // codes, or what they are made from
  long bs, rs;
  const float* xscale;         // of codes
  char* out;
  int T, P, K, M, pitch;
  float floor;
};

// NT: tiles of 16 tokens, MT: of 16 weight rows.  DT: the type the codes are
// made from here, or 3: codes already.
template <int DT, int OUT, int NT, int MT>
__global__ __launch_bounds__(kThreads) void k_mix_i8_few(Args p) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ uint32_t tops[16 * NT];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = blockIdx.x * 16 * MT, blocks = p.pitch / 128;
  if constexpr (DT == 3) {   // this block's tokens
    const int t0 = blockIdx.y * 16 * NT;
    p.x += (long)t0 * p.pitch;
    p.xscale += t0;
    p.out += (long)t0 * p.M * kBytes<OUT>;
    p.T = min(p.T - t0, 16 * NT);
  }
  // chunk 4 s + lane / 16 of row lane % 16 in matrix instruction s of a block
  typedef i32x4_t Weights[MT][kAhead][2];
  Weights a;
  auto load_w = [&](Weights& a, int first) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (first + u * kWaves >= blocks) break;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int8_t* w = p.w + (long)min(m0 + 16 * m + (lane & 15), p.M - 1) * p.pitch + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < 2; ++s)
          a[m][u][s] = *reinterpret_cast<const i32x4_t*>(w + (first + u * kWaves) * 128 + s * 64);
      }
    }
  };
  load_w(a, wave);

  // codes of token t at smem + t * row (+ 16: 16 tokens' reads hit all banks)
  const int row = p.pitch + 16;
  float* scales = reinterpret_cast<float*>(smem + (DT == 3 ? 0 : p.T * row));   // then the waves' sums
  if constexpr (DT != 3) {
    const int per = (p.K + 511) / 512, items = p.T * per;   // pieces of a token, in all
    Raw<kWords<DT, 8>> x[kItems];
    if (tid < 16 * NT) tops[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int it = wave + i * kWaves, t = it / per, k = (it % per) * 512 + lane * 8;
      const char* at = p.x + ((long)(t / p.P) * p.bs + (long)(t % p.P) * p.rs + k) * kBytes<DT>;
      x[i] = Raw<kWords<DT, 8>>{};
      if (p.K % 512 == 0) {   // whole pieces
        if (it < items) x[i] = load_wide<DT, 8>(at);
      } else {
        x[i] = load_vec<DT, 8>(at, it < items ? p.K - k : 0);
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int it = wave + i * kWaves;
      if (it >= items) break;
      Largest<DT, 8> largest;
      largest.take(x[i]);
      uint32_t top = largest.all();
#pragma unroll
      for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      if (lane == 0) atomicMax(&tops[it / per], top);   // the largest: in any order
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int it = wave + i * kWaves;
      if (it >= items) break;
      const int t = it / per, k = (it % per) * 512 + lane * 8;
      const float inv = row_scale(tops[t]).inv;
      if (k < p.pitch) {
        Raw<2> q;
        q[0] = codes4(elem<DT, 8>(x[i], 0), elem<DT, 8>(x[i], 1), elem<DT, 8>(x[i], 2), elem<DT, 8>(x[i], 3), inv);
        q[1] = codes4(elem<DT, 8>(x[i], 4), elem<DT, 8>(x[i], 5), elem<DT, 8>(x[i], 6), elem<DT, 8>(x[i], 7), inv);
        *reinterpret_cast<Raw<2>*>(smem + t * row + k) = q;
      }
    }
    __syncthreads();
    if (tid < p.T) scales[tid] = row_scale(tops[tid]).scale;
  } else {
    if (tid < p.T) scales[tid] = p.xscale[tid];
  }

  i32x4_t acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = i32x4_t{0, 0, 0, 0};
  auto multiply = [&](const Weights& a, int first) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int t = min(16 * n + (lane & 15), p.T - 1);
      i32x4_t b[kAhead][2];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (first + u * kWaves >= blocks) break;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int at = (first + u * kWaves) * 128 + s * 64 + (lane >> 4) * 16;
          if constexpr (DT == 3) b[u][s] = *reinterpret_cast<const i32x4_t*>(p.x + (long)t * p.pitch + at);
          else b[u][s] = *reinterpret_cast<const i32x4_t*>(smem + t * row + at);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (first + u * kWaves >= blocks) break;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[m][u][s], b[u][s], acc[m][n], 0, 0, 0);
      }
    }
  };
  constexpr int kRound = kAhead * kWaves;   // blocks that the waves load together
  if constexpr (MT == 2) {
    multiply(a, wave);   // all of them (launch)
  } else {
    Weights c;
    for (int first = wave; first < blocks; first += 2 * kRound) {
      load_w(c, first + kRound);
      multiply(a, first);
      load_w(a, first + 2 * kRound);
      multiply(c, first + kRound);
    }
  }
  // sums of the waves: element r of a lane is weight row 4 (lane / 16) + r,
  // token lane % 16
  int* sums = reinterpret_cast<int*>(scales + 16 * NT);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      *reinterpret_cast<i32x4_t*>(sums + (((wave * NT + n) * MT + m) * 64 + lane) * 4) = acc[m][n];
  __syncthreads();
  for (int o = tid; o < NT * MT * 256; o += kThreads) {
    const int m = o % (16 * MT), t = o / (16 * MT);   // weight rows of a token side by side
    if (m0 + m >= p.M || t >= p.T) continue;
    const int at = (((t >> 4) * MT + (m >> 4)) * 64 + (m >> 2 & 3) * 16 + (t & 15)) * 4 + (m & 3);
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) sum += sums[k * NT * MT * 256 + at];
    const float v = __fmaf_rn((float)sum * scales[t], p.wscale[m0 + m], p.bias ? p.bias[m0 + m] : 0.f);
    const float z = v < p.floor ? p.floor : v;   // a NaN stays
    const long to = (long)t * p.M + m0 + m;
    if constexpr (OUT == kBF16) reinterpret_cast<uint16_t*>(p.out)[to] = (uint16_t)pair_bf16(z, 0.f);
    else reinterpret_cast<float*>(p.out)[to] = z;
  }
}

long blocks_of(int M, int m, long T, int t) { return (long)((M + m - 1) / m) * ((T + t - 1) / t); }

template <int DT, int OUT, int MT>
hipError_t launch_rows(const Args& p, hipStream_t s) {
  // tiles of tokens to a block: of codes as few as leave one block to a CU (200
  // tokens 4096 -> 256: 6.2 us, with three each 9.8; 64 tokens 8192 -> 512: 9.8, 17)
  int nt = min((p.T + 15) / 16, DT == 3 ? 3 : 2);
  if (DT == 3)
    for (int n = nt - 1; n > 0; --n)
      if (blocks_of(p.M, 16 * MT, p.T, 16 * n) <= 256) nt = n;
  const size_t lds = (DT == 3 ? 0 : (size_t)p.T * (p.pitch + 16)) + (size_t)nt * (64 + kWaves * MT * 1024);
  const dim3 grid((unsigned)((p.M + 16 * MT - 1) / (16 * MT)), (unsigned)((p.T + 16 * nt - 1) / (16 * nt)));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, s, p); };
  switch (nt) {
    case 1: go(k_mix_i8_few<DT, OUT, 1, MT>); break;
    case 2: go(k_mix_i8_few<DT, OUT, 2, MT>); break;
    default:   // codes made in the block: at most two tiles
      if constexpr (DT == 3) go(k_mix_i8_few<DT, OUT, 3, MT>);
  }
  return hipGetLastError();
}

// Two tiles of weight rows to a block, which halves the tokens' reads, where
// that leaves a block per CU and one round of loads: kernel us with one and
// two, 24 tokens 2048 -> 8192: 7.5, 6.9; 1 token 4096 -> 8192: 8.9, 8.6; 8
// tokens 4096 -> 4096: 5.7, 7.7; 4 tokens 8192 -> 8192: 15.4, 20.2 (two rounds).
template <int DT, int OUT>
hipError_t launch(const Args& p, hipStream_t s) {
  const bool two = p.M >= 8192 && p.pitch <= kAhead * kWaves * 128;
  return two ? launch_rows<DT, OUT, 2>(p, s) : launch_rows<DT, OUT, 1>(p, s);
}

}  // namespace

// Against the tiles of bc_mix_i8.hip, kernel us: 8 tokens 4096 -> 4096 5.7 and
// 13.7, 32 tokens 8.6 and 13.9, 48 10.6 and 13.8, 64 tokens 4096 -> 8192 15.9
// and 14.5, 33 tokens 8192 -> 8192 26.5 and 24.6: the tokens' codes, read by
// every block, take over.  Where few weight rows leave a CU no more than a block:
// 64 tokens 4096 -> 1024 6.3 and 12.3, 600 tokens 4096 -> 256 10.2 and 12.4, 200
// tokens 8192 -> 512 13.6 and 20; past it 100 tokens 2048 -> 2048 8.8 and 8.2.
bool mix_i8_few_takes(long rows, int K, int M) {
  return rows <= (K <= 4096 ? 48 : 32) || blocks_of(M, 16, rows, 48) <= 256;
}

// In the block: pieces of 512 values, kItems for each wave.
bool mix_i8_few_makes_codes(long rows, int K) { return rows <= 32 && rows * ((K + 511) / 512) <= kItems * kWaves; }

hipError_t launch_mix_i8_few(const MixI8& m, hipStream_t s) {
  Args p{};
  p.w = static_cast<const int8_t*>(m.wq);
  p.wscale = m.wscale;
  p.bias = m.bias;
  p.x = static_cast<const char*>(m.x);
  p.bs = m.bs;
  p.rs = m.rs;
  p.xscale = m.xscale;
  p.out = static_cast<char*>(m.out);
  p.T = m.N * m.P;
  p.P = m.P;
  p.K = m.K;
  p.M = m.M;
  p.pitch = i8_pitch(m.K);
  p.floor = m.relu ? 0.f : -INFINITY;
  const bool bf16 = m.out_dt == kBF16;
  if (m.dt == 3) return bf16 ? launch<3, kBF16>(p, s) : launch<3, kF32>(p, s);
  if (m.dt == kBF16) return bf16 ? launch<kBF16, kBF16>(p, s) : launch<kBF16, kF32>(p, s);
  return bf16 ? launch<kF32, kBF16>(p, s) : launch<kF32, kF32>(p, s);
}

}  // namespace bc
