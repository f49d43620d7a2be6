// The 1x1 mix in 8-bit codes on maps [N][K][P], codes and product in one pass
// (gfx950; bc_i8.hpp has the codes' definition).
//
// Bound by memory: maps in, maps out, and little arithmetic for them (M is a
// few hundred).  A block takes 64 (or 32) pixels of one image by all K channels:
// it reads them once, keeping them in registers until the pixels' scales are
// known (as many as fit; the rest is read again), turns the codes through LDS
// into the rows that the matrix instructions read, and multiplies them with all
// M weight rows, which come from the XCD's L2.  The codes never go to memory.
// 32 images of 1024 x 64 x 64 bf16 to 256 fp32 maps: 111 us with other tensors in
// every call, 403 MB at 3.6 TB/s (90 with the same); codes and products take a
// third of it, in which the block's loads stand still.
#include "bc_i8.hpp"

#include <math.h>

#include <type_traits>

namespace bc {
namespace {

using namespace i8;

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

struct Args {
  const char* x;
  long bs, rs;
  const int8_t* w;
  const float *wscale, *bias;
  char* out;
  int M, K, P, pitch, strips, steps, packed;
  bool near;
  float floor;
};

// kLined: past the caches.
template <int OUT, bool kLined>
__device__ __forceinline__ void store_one(char* o, float z) {
  typedef typename std::conditional<OUT == kBF16, uint16_t, float>::type T;
  T v;
  if constexpr (OUT == kBF16) v = (uint16_t)pair_bf16(z, 0.f);
  else v = z;
  if constexpr (kLined) __builtin_nontemporal_store(v, reinterpret_cast<T*>(o));
  else *reinterpret_cast<T*>(o) = v;
}

template <int DT, int OUT, int PX, bool kLined, int kHold, bool kFull>
__device__ __forceinline__ void mix_tile(const Args& p, int n, int pt, uint32_t lds, uint32_t* tops, RowScale* rows) {
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int XB = PX / 32;   // blocks of 32 pixels
  const Pixels at(tid % (PX / 8) * 8, p.P - pt, p.P);
  const int lp = p.steps * kStepK<PX>;
  const char* base = p.x + ((long)n * p.bs + pt + at.first) * kBytes<DT>;
  // a wave: 32 weight rows by the pixels.  Lane l of matrix instruction t of a
  // block of 128 codes has chunk 2 t + l / 32 of row l % 32.
  const int pa = lane & 31, blocks = p.pitch / 128;
  const int wt = p.packed ? 1024 : 32, wk = 4 * wt;   // bytes from one t to the next, from a block to the next
  auto weights = [&](int m0) {
    return p.packed ? p.w + (long)m0 * p.pitch + lane * 16
                    : p.w + (long)min(m0 + pa, p.M - 1) * p.pitch + half * 16;
  };
  i32x4_t b[4], next[4];
  auto first = [&](int m0) {
    const int8_t* w = weights(m0);
#pragma unroll
    for (int t = 0; t < 4; ++t) b[t] = *reinterpret_cast<const i32x4_t*>(w + t * wt);
  };
  {
    Raw<kWords<DT, 8>> x[kHold + 1][4];
    tile_scales<DT, PX, kHold, kFull>(base, p.rs, at, p.K, x, tops, rows);
    if (wave * 32 < p.M) first(wave * 32);   // on its way while the codes are made
    tile_codes<DT, PX, kHold, kFull>(base, p.rs, at, p.K, x, rows, lds, lp, 0, p.steps);
  }
  __syncthreads();
  const int swap[2] = {chunk_swap<PX>(pa), chunk_swap<PX>(pa + 32)};
  for (int m0 = wave * 32; m0 < p.M; m0 += kTileThreads / 64 * 32) {
    if (m0 > wave * 32) first(m0);
    const int8_t* w = weights(m0);
    // scales and biases of the lane's rows: element r of a lane is weight row
    // 8 (r / 4) + 4 half + r % 4.  Ahead of the products where registers are left.
    constexpr bool kEarly = XB == 1;
    float sw[16], bias[16];
    auto row_factors = [&]() {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int mr = min(m0 + 8 * (r >> 2) + 4 * half + (r & 3), p.M - 1);
        sw[r] = p.wscale[mr];
        bias[r] = p.bias ? p.bias[mr] : 0.f;
      }
    };
    if (kEarly) row_factors();
    i32x16_t acc[XB];
#pragma unroll
    for (int x = 0; x < XB; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][r] = 0;
    for (int k = 0; k < blocks; ++k) {
      if (k + 1 < blocks) w += wk;   // the last block again: never used
#pragma unroll
      for (int t = 0; t < 4; ++t) next[t] = *reinterpret_cast<const i32x4_t*>(w + t * wt);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < XB; ++x) {
          const int c = k * 8 + 2 * t + half;
          const i32x4_t a = *(BC_LDS i32x4_t*)(uintptr_t)(lds + (pa + 32 * x) * lp + ((c ^ swap[x]) << 4));
          acc[x] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[t], a, acc[x], 0, 0, 0);
        }
#pragma unroll
      for (int t = 0; t < 4; ++t) b[t] = next[t];
    }
    if (!kEarly) row_factors();
    // a store writes 32 pixels of a row in one run
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int mr = m0 + 8 * (r >> 2) + 4 * half + (r & 3);
      if (mr >= p.M) continue;
      char* o = p.out + (((long)n * p.M + mr) * p.P + pt + pa) * kBytes<OUT>;
#pragma unroll
      for (int x = 0; x < XB; ++x) {
        const float v = __fmaf_rn((float)acc[x][r] * rows[pa + 32 * x].scale, sw[r], bias[r]);
        const float z = v < p.floor ? p.floor : v;   // a NaN stays
        if (!kFull && pt + pa + 32 * x >= p.P) continue;
        store_one<OUT, kLined>(o + 32 * x * kBytes<OUT>, z);
      }
    }
  }
}

// kLined: outputs go past the caches, where their rows are whole runs of 16 bytes;
// others' shared pieces are put together in an L2.  Where rows are not whole 64
// bytes, neighbouring strips go to one XCD (18 images of 160 x 7469 to 383 fp32
// maps: 119 us past the caches in order, 105 through them, 89 with neighbours;
// rows of 7464 bf16 past the caches 75 and 68; rows of 7472 fp32 67 and 77).
template <int DT, int OUT, int PX, bool kLined>
__global__ __launch_bounds__(kTileThreads, 4) void k_mix_i8_maps(Args p) {
  extern __shared__ __align__(16) unsigned char smem[];   // codes of the pixels
  __shared__ uint32_t tops[kTileThreads / 64 * PX];
  __shared__ RowScale rows[PX];
  const int b = tile_of_block(p.near);
  const int n = b / p.strips, pt = (b % p.strips) * PX;
  const uint32_t lds = (uint32_t)(uintptr_t)(BC_LDS unsigned char*)smem;
  if (p.P - pt >= PX) mix_tile<DT, OUT, PX, kLined, kHeld<DT>, true>(p, n, pt, lds, tops, rows);
  else mix_tile<DT, OUT, PX, kLined, kHeld<DT>, false>(p, n, pt, lds, tops, rows);
}

// Weight rows in the order in which the waves read them: 32 rows by 128 codes at
// a time, 4 matrix instructions, 64 lanes, 16 bytes.  A wave's load is then 1
// KiB in one piece, where rows as they are cost it 32 cache lines.
__global__ __launch_bounds__(256) void k_pack_rows(const int8_t* w, i32x4_t* out, int M, int pitch, long chunks) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int lane = (int)(i & 63), t = (int)(i >> 6) & 3;
  const long block = i >> 8;   // of 32 x 128 codes
  const int per = pitch / 128, m = min((int)(block / per) * 32 + (lane & 31), M - 1);
  const int k = (int)(block % per) * 128 + (2 * t + (lane >> 5)) * 16;
  out[i] = *reinterpret_cast<const i32x4_t*>(w + (long)m * pitch + k);
}

long strips_of(int N, int P, int px) { return (long)N * ((P + px - 1) / px); }

// Pixels of a block.  64 read the weights half as often as 32 (32 images of 1024
// x 64 x 64 to 256 maps: 95 and 147 us); 32 make twice the blocks where there
// are few (1 x 1024 x 64 x 64 to 256: 14.4 and 12.6), and leave room for two on a
// CU where a pixel's codes are many and the weight rows few (16 x 2048 x 1000 to
// 200: 48 and 43; 2 x 2048 x 8000 to 1024: 67 and 74).
bool wide_blocks(int N, int M, int K, int P) {
  return strips_of(N, P, 64) >= 256 && (K <= 1024 || M > 512);
}

// Blocks from which the packing's launch pays (32 images of 1024 x 64 x 64 to
// 256 maps: 124 us without, 95 + 5 with; 64 blocks 33 and 32).
constexpr long kPackBlocks = 32;

template <int DT, int OUT, int PX, bool kLined>
hipError_t launch(Args& p, int N, hipStream_t s) {
  p.strips = (p.P + PX - 1) / PX;
  p.steps = (p.pitch + kStepK<PX> - 1) / kStepK<PX>;
  const size_t lds = (size_t)PX * p.steps * kStepK<PX>;
  hipLaunchKernelGGL((k_mix_i8_maps<DT, OUT, PX, kLined>), dim3((unsigned)((long)N * p.strips)), dim3(kTileThreads), lds, s, p);
  return hipGetLastError();
}

template <int DT, int OUT>
hipError_t launch(Args& p, int N, hipStream_t s) {
  const bool lined = (long)p.P * kBytes<OUT> % 16 == 0 && (uintptr_t)p.out % 16 == 0;
  if (wide_blocks(N, p.M, p.K, p.P)) return lined ? launch<DT, OUT, 64, true>(p, N, s) : launch<DT, OUT, 64, false>(p, N, s);
  return lined ? launch<DT, OUT, 32, true>(p, N, s) : launch<DT, OUT, 32, false>(p, N, s);
}

}  // namespace

// Not the calls whose few pixels meet many weight rows: the tiles of
// bc_mix_i8.hip divide those over the chip (kernel us here and there: 1 x 2000 x
// 500 to 1000 79 and 20, 4 x 2048 x 1000 to 1024 51 and 38; 1 x 1024 x 64 x 64 to
// 256 15 and 19).
bool mix_i8_maps_takes(int N, int M, int K, int P) {
  return K <= 2048 && (M <= 256 || strips_of(N, P, 64) >= 128);
}

size_t mix_i8_maps_workspace_bytes(int N, int M, int K, int P) {
  return strips_of(N, P, 64) < kPackBlocks ? 0 : (size_t)(M + 31) / 32 * 32 * i8_pitch(K);
}

hipError_t launch_mix_i8_maps(const MixI8& m, hipStream_t s) {
  Args p{};
  p.x = static_cast<const char*>(m.x);
  p.bs = m.bs;
  p.rs = m.rs;
  p.w = static_cast<const int8_t*>(m.wq);
  p.wscale = m.wscale;
  p.bias = m.bias;
  p.out = static_cast<char*>(m.out);
  p.M = m.M;
  p.K = m.K;
  p.P = m.P;
  p.pitch = i8_pitch(m.K);
  p.floor = m.relu ? 0.f : -INFINITY;
  p.near = (long)m.P * (m.out_dt == kBF16 ? 2 : 4) % 64 != 0;
  const size_t packed = mix_i8_maps_workspace_bytes(m.N, m.M, m.K, m.P);
  if (packed > 0) {
    const long chunks = (long)packed / 16;
    hipLaunchKernelGGL(k_pack_rows, dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, s, p.w,
                       static_cast<i32x4_t*>(m.ws), p.M, p.pitch, chunks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.w = static_cast<const int8_t*>(m.ws);
    p.packed = 1;
  }
  if (m.dt == kBF16) return m.out_dt == kBF16 ? launch<kBF16, kBF16>(p, m.N, s) : launch<kBF16, kF32>(p, m.N, s);
  return m.out_dt == kBF16 ? launch<kF32, kBF16>(p, m.N, s) : launch<kF32, kF32>(p, m.N, s);
}

}  // namespace bc
