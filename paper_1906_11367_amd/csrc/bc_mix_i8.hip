// The 1x1 mix of 8-bit codes (gfx950): out = (codes of a token . codes of a
// weight row) * token scale * weight scale + bias, the product exact in int32.
// Both operands are rows contiguous along the reduction, padded with zeros to
// whole 128 bytes; rows i of one and rows j of the other give out(i, j), i the
// index that is contiguous in the output: tokens [T][M] take i = weight row,
// j = token, maps [N][M][P] the reverse.
// Bound by the matrix instructions where the sizes are large: 16384 x 4096 to
// 8192 takes 490 to 540 us with the clocks' state (2250 to 2040 TOP/s; the
// vendor's library 480 to 500).  Sizes that 256 x 256 tiles leave most CUs idle at
// take smaller ones, up to twice as slow for each product (launch): 1024 x 4096
// to 4096, one round of 256 tiles of 128 x 128, 26 us (1330 TOP/s).
#include "bc_internal.hpp"
#include "bc_scan.hpp"

#include <math.h>

#include <algorithm>

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
  int pitch, M, P;
  float floor;                // 0 with relu, else -infinity
  bool stream;                // out past the caches (bc_scan.hpp: streams)
};

// Where out(i, j) stands, in elements.
template <bool kMaps>
__device__ __forceinline__ long out_at(const Args& p, int i, int j) {
  if constexpr (kMaps) return ((long)(i / p.P) * p.M + j) * p.P + i % p.P;
  else return (long)j * p.M + i;
}

__device__ __forceinline__ float finish(int sum, float token, float weight, float bias, float floor) {
  const float z = __fmaf_rn((float)sum * token, weight, bias);
  return z < floor ? floor : z;   // a NaN stays
}

#define BC_LDS __attribute__((address_space(3)))

__device__ __forceinline__ i32x4_t buf_desc(const void* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)p;
  i32x4_t r;
  r.x = __builtin_amdgcn_readfirstlane((int)a);
  r.y = __builtin_amdgcn_readfirstlane((int)(a >> 32));
  r.z = __builtin_amdgcn_readfirstlane((int)bytes);
  r.w = 0x00020000;
  return r;
}

// 16 bytes per lane from (desc, voff + soff) to LDS at lds + 16 * lane, waited
// for by count (wait_loads).
__device__ __forceinline__ void load_to_lds(const i32x4_t& rs, uint32_t voff, uint32_t soff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 1\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               ::"s"(lds), "v"(voff), "s"(rs), "s"(soff)
               : "memory", "m0");
}

// Waits until at most kLeft of the wave's loads are pending, and for its LDS
// reads (whose place the loads after the next barrier may take).
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");
}

// Tiles through LDS: WI x WJ waves of FI x FJ blocks of 32 x 32 outputs.
//
// Both operands go from memory into a ring of LDS stages (kBK codes, 64 or 128,
// of every row of the tile), kStages - 1 stages ahead, one barrier per stage.
// The 16-byte chunk c of row r sits at chunk c ^ chunk_of(r), so that the 16
// lanes that read one chunk of 16 rows hit all banks; the loads write LDS in
// lane order, so each lane fetches the chunk that belongs there.
template <int kBK>
__device__ __forceinline__ int chunk_of(int r) { return kBK == 64 ? (r >> 2) & 3 : (r >> 1) & 7; }

template <int OUT, bool kMaps, int WI, int WJ, int FI, int FJ, int kBK, int kStages>
__global__ __launch_bounds__(64 * WI * WJ) void k_mix_i8_tile(Args p, int ti, int tj, int per) {
  constexpr int kWaves = WI * WJ, BI = WI * FI * 32, BJ = WJ * FJ * 32;
  constexpr int kABytes = BI * kBK, kStage = (BI + BJ) * kBK;
  constexpr int kALoads = kABytes / 1024, kLoads = kStage / 1024 / kWaves;   // kLoads: per wave
  static_assert(kStage % (1024 * kWaves) == 0, "whole loads");
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(BC_LDS unsigned char*)smem;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // consecutive tiles on one XCD; 8 tiles of i for each of j, so that the
  // tiles running together share both operands in its L2
  const int L = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (L >= ti * tj) return;
  const int grp = L / (8 * tj), in = L - grp * 8 * tj, gsz = min(8, ti - grp * 8);
  const int i0 = (grp * 8 + in % gsz) * BI, j0 = in / gsz * BJ;
  const int nk = p.pitch / kBK;
  const i32x4_t ra = buf_desc(p.a + (long)i0 * p.pitch, (uint32_t)(min(BI, p.I - i0) * p.pitch));
  const i32x4_t rb = buf_desc(p.b + (long)j0 * p.pitch, (uint32_t)(min(BJ, p.J - j0) * p.pitch));

  uint32_t voff[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int ld = wave * kLoads + l;
    const bool is_a = ld < kALoads;
    constexpr int kLanes = kBK / 16, kLoadRows = 64 / kLanes;   // lanes on a row, rows of a load
    const int row = (is_a ? ld : ld - kALoads) * kLoadRows + lane / kLanes;
    // rows past the operand read zeros (the descriptor ends there)
    voff[l] = (uint32_t)row * (uint32_t)p.pitch + (uint32_t)(((lane & (kLanes - 1)) ^ chunk_of<kBK>(row)) * 16);
  }
  int load_slot = 0, load_k = 0;
  auto issue = [&]() {
    const uint32_t base = lds0 + load_slot * kStage;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int ld = wave * kLoads + l;
      load_to_lds(ld < kALoads ? ra : rb, voff[l], (uint32_t)(load_k * kBK), base + ld * 1024);
    }
    load_slot = load_slot + 1 == kStages ? 0 : load_slot + 1;
    ++load_k;
  };

  const int wi = wave / WJ, wj = wave % WJ;
  // rows 32 apart swizzle alike
  const int arow = wi * FI * 32 + (lane & 31), brow = wj * FJ * 32 + (lane & 31);
  constexpr int kSteps = kBK / 32;   // matrix instructions deep
  uint32_t aoff[kSteps], boff[kSteps];
#pragma unroll
  for (int kk = 0; kk < kSteps; ++kk) {
    const int c = 2 * kk + (lane >> 5);
    aoff[kk] = (uint32_t)(arow * kBK + ((c ^ chunk_of<kBK>(arow)) << 4));
    boff[kk] = (uint32_t)(kABytes + brow * kBK + ((c ^ chunk_of<kBK>(brow)) << 4));
  }
  i32x16_t acc[FI][FJ];
#pragma unroll
  for (int x = 0; x < FI; ++x)
#pragma unroll
    for (int y = 0; y < FJ; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0;

  // A stage is kSteps steps of 32 codes.  The operands of a step are read from
  // LDS during the step before, across the barrier too, which stands before a
  // stage's last step: no wave then starts a stage by waiting for its reads.
  i32x4_t fa[2][FI], fb[2][FJ];
  auto read = [&](int step, uint32_t st) {
    const int half = step & 1;
#pragma unroll
    for (int x = 0; x < FI; ++x) fa[half][x] = *(BC_LDS i32x4_t*)(uintptr_t)(st + aoff[step] + x * 32 * kBK);
#pragma unroll
    for (int y = 0; y < FJ; ++y) fb[half][y] = *(BC_LDS i32x4_t*)(uintptr_t)(st + boff[step] + y * 32 * kBK);
  };
  auto multiply = [&](int step) {
    const int half = step & 1;
#pragma unroll
    for (int x = 0; x < FI; ++x)
#pragma unroll
      for (int y = 0; y < FJ; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[half][x], fb[half][y], acc[x][y], 0, 0, 0);
  };
  // the reads spread over the matrix instructions
  auto interleave = [&]() {
#pragma unroll
    for (int k = 0; k < (FI * FJ > FI + FJ ? FI * FJ : FI + FJ); ++k) {
      if (k < FI * FJ) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (k < FI + FJ) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
  };
  for (int s = 0; s < kStages - 1 && s < nk; ++s) issue();
  if (nk >= kStages - 1) wait_loads<kLoads * (kStages - 2)>();
  else wait_loads<0>();
  __builtin_amdgcn_s_barrier();
  read(0, lds0);
  int slot = 0;
  for (int s = 0; s < nk; ++s) {
    const uint32_t st = lds0 + slot * kStage;
#pragma unroll
    for (int step = 0; step + 1 < kSteps; ++step) {
      __builtin_amdgcn_sched_barrier(0);
      read(step + 1, st);
      multiply(step);
      interleave();
    }
    __builtin_amdgcn_sched_barrier(0);
    // the next stage's loads are done when at most the later ones' are pending
    if (s + kStages - 2 < nk) wait_loads<kLoads * (kStages - 3)>();
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (load_k < nk) issue();
    slot = slot + 1 == kStages ? 0 : slot + 1;
    read(0, lds0 + slot * kStage);   // past the last stage: never used
    multiply(kSteps - 1);
    interleave();
  }
  __builtin_amdgcn_sched_barrier(0);

  // Outputs.  A lane holds, of column j = lane % 32 of a block, rows 8 (r / 4) +
  // 4 (lane / 32) + r % 4: four consecutive i at a time.  They go through the
  // wave's own part of LDS, 32 columns j at a time, to be stored 16 bytes a lane
  // along i.
  constexpr int kE = kBytes<OUT>, kWide = 16 / kE, kRow = FI * 32 * kE + 16;   // + 16: lanes hit distinct banks
  const int ib = i0 + wi * FI * 32, jb = j0 + wj * FJ * 32;
  const uint32_t mine = lds0 + wave * 32 * kRow;
  float* iscale = reinterpret_cast<float*>(smem + kWaves * 32 * kRow);   // and the biases after the scales
  __syncthreads();   // the stages are read
  for (int i = threadIdx.x; i < BI; i += 64 * kWaves) {
    const int at = min(i0 + i, p.I - 1);
    iscale[i] = p.ascale[at];
    iscale[BI + i] = !kMaps && p.bias ? p.bias[at] : 0.f;
  }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < FJ; ++y) {
    const int j = min(jb + 32 * y + (lane & 31), p.J - 1);
    const float sj = p.bscale[j], bj = kMaps && p.bias ? p.bias[j] : 0.f;
#pragma unroll
    for (int x = 0; x < FI; ++x)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float* si = iscale + wi * FI * 32 + 32 * x + 8 * g + 4 * (lane >> 5);
        float z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          z[k] = kMaps ? finish(acc[x][y][4 * g + k], si[k], sj, bj, p.floor)
                       : finish(acc[x][y][4 * g + k], sj, si[k], si[BI + k], p.floor);
        const uint32_t at = mine + (lane & 31) * kRow + (32 * x + 8 * g + 4 * (lane >> 5)) * kE;
        if constexpr (OUT == kBF16) {
          const Raw<2> w = {pair_bf16(z[0], z[1]), pair_bf16(z[2], z[3])};
          *(BC_LDS Raw<2>*)(uintptr_t)at = w;
        } else {
          const Raw<4> w = {__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])};
          *(BC_LDS Raw<4>*)(uintptr_t)at = w;
        }
      }
    constexpr int kChunks = FI * 32 / kWide;   // 16-byte chunks of a column j
    static_assert(32 * kChunks % 64 == 0, "whole waves of chunks");
#pragma unroll
    for (int c0 = 0; c0 < 32 * kChunks; c0 += 64) {
      const int c = c0 + lane, jj = c / kChunks, ii = c % kChunks * kWide;
      const Raw<4> w = *(BC_LDS Raw<4>*)(uintptr_t)(mine + jj * kRow + ii * kE);
      const int i = ib + ii, jo = jb + 32 * y + jj;
      if (i >= p.I || jo >= p.J) continue;
      char* o = p.out + out_at<kMaps>(p, i, jo) * kE;
      const int left = kMaps ? min(p.I - i, p.P - i % p.P) : p.I - i;   // elements contiguous from here
      if (left >= kWide && p.stream) {
        typedef Raw<kWide * kE / 4> Any __attribute__((aligned(kE)));
        asm volatile("");   // keeps the compiler from merging the two stores into a plain one
        __builtin_nontemporal_store(w, reinterpret_cast<Any*>(o));
        asm volatile("");
      } else if (left >= kWide) {
        *reinterpret_cast<Loose<4, kE>*>(o) = __builtin_bit_cast(Loose<4, kE>, w);
      } else {
#pragma unroll
        for (int k = 0; k < kWide; ++k) {
          if (i + k >= p.I) break;
          char* e = p.out + out_at<kMaps>(p, i + k, jo) * kE;
          if constexpr (OUT == kBF16) *reinterpret_cast<uint16_t*>(e) = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
          else *reinterpret_cast<uint32_t*>(e) = w[k];
        }
      }
    }
  }
}

template <int OUT, bool kMaps, int WI, int WJ, int FI, int FJ, int kBK, int kStages>
hipError_t launch_tile(const Args& p, hipStream_t s) {
  constexpr int BI = WI * FI * 32, BJ = WJ * FJ * 32;
  constexpr int kLds = std::max(kStages * (BI + BJ) * kBK, WI * WJ * 32 * (FI * 32 * kBytes<OUT> + 16) + BI * 8);
  const auto kernel = k_mix_i8_tile<OUT, kMaps, WI, WJ, FI, FJ, kBK, kStages>;
  const int ti = (p.I + BI - 1) / BI, tj = (p.J + BJ - 1) / BJ, per = (ti * tj + 7) / 8;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(per * 8)), dim3(64 * WI * WJ), kLds, s, p, ti, tj, per);
  return hipGetLastError();
}

// Tiles, and the time of a round of them on 256 CUs for 4096 codes (us): wide tiles
// read their operands less often, narrow ones leave fewer CUs idle in the last
// round.  Stages of 128 codes halve the barriers where LDS has room for them.
//   256 x 256        one to a CU       54
//   256 x 128        one               34
//   128 x 128        two               46 (28 for one)
//   128 x 128, deep  one               26
//   64 x 64          two               15.5 (14)
// The least sum of rounds is the fastest or within 5 % at 37 sizes measured; kernel
// us in the order above:
//   2048 x 8192 -> 8192  128,  160,  184,  165,  228
//   2048 x 4096 -> 4096  53.9, 38.3, 46.5, 47.5, 58.6
//   1337 x 3495 -> 6448  51.5, 59.6, 59.3, 60.6, 60.7
//   1500 x 2000 -> 3000  32.1, 22.0, 23.4, 27.8, 24.4
//   1024 x 4096 -> 4096  51.8, 33.4, 28.2, 25.8, 31.2
//   751 x 2552 -> 5380   37.7, 26.8, 30.0, 33.0, 24.4
//   512 x 4096 -> 4096   48.8, 31.6, 25.2, 22.6, 17.5
template <int OUT, bool kMaps>
hipError_t launch(const Args& p, hipStream_t s) {
  auto tiles = [&](int i, int j) { return (long)((p.I + i - 1) / i) * ((p.J + j - 1) / j); };
  // pairs of tiles to a CU; the last round may have one
  auto pairs = [](long t, long two, long one) { return t / 512 * two + (t % 512 > 256 ? two : t % 512 > 0 ? one : 0); };
  const long c128 = tiles(128, 128);
  const long cost[5] = {(tiles(256, 256) + 255) / 256 * 540, (tiles(256, 128) + 255) / 256 * 340, pairs(c128, 460, 280),
                        (c128 + 255) / 256 * 260, pairs(tiles(64, 64), 155, 140)};
  switch (std::min_element(cost, cost + 5) - cost) {
    case 0: return launch_tile<OUT, kMaps, 2, 4, 4, 2, 64, 4>(p, s);
    case 1: return launch_tile<OUT, kMaps, 4, 2, 2, 2, 128, 3>(p, s);
    case 2: return launch_tile<OUT, kMaps, 2, 2, 2, 2, 64, 4>(p, s);
    case 3: return launch_tile<OUT, kMaps, 2, 2, 2, 2, 128, 4>(p, s);
    default: return launch_tile<OUT, kMaps, 2, 2, 1, 1, 128, 4>(p, s);
  }
}

// Workspace: the tokens' codes, then their scales.
size_t codes_bytes(long rows, int K) { return ((size_t)rows * i8_pitch(K) + 255) & ~(size_t)255; }

}  // namespace

size_t mix_i8_workspace_bytes(int N, int M, int K, int P, int dt, bool maps) {
  if (dt == 3) return 0;   // codes already
  if (maps && mix_i8_maps_takes(N, M, K, P)) return mix_i8_maps_workspace_bytes(N, M, K, P);
  const long rows = (long)N * P;
  if (!maps && mix_i8_few_makes_codes(rows, K)) return 0;
  return codes_bytes(rows, K) + (size_t)rows * 4;
}

hipError_t launch_mix_i8(const MixI8& m, hipStream_t s) {
  if (m.maps && m.dt != 3 && mix_i8_maps_takes(m.N, m.M, m.K, m.P)) return launch_mix_i8_maps(m, s);
  const long rows = (long)m.N * m.P;
  const bool few = !m.maps && mix_i8_few_takes(rows, m.K, m.M);
  const int8_t* x = static_cast<const int8_t*>(m.x);
  const float* xscale = m.xscale;
  if (few && (m.dt == 3 || mix_i8_few_makes_codes(rows, m.K))) return launch_mix_i8_few(m, s);
  if (m.dt != 3) {
    char* ws = static_cast<char*>(m.ws);
    float* scale = reinterpret_cast<float*>(ws + codes_bytes(rows, m.K));
    const hipError_t e = launch_quantize_i8(m.x, m.dt, m.bs, m.rs, ws, scale, m.N, m.K, m.P, m.maps, s);
    if (e != hipSuccess) return e;
    x = reinterpret_cast<const int8_t*>(ws);
    xscale = scale;
  }
  if (few) {
    MixI8 c = m;
    c.x = x;
    c.xscale = xscale;
    c.dt = 3;
    c.N = 1;
    c.P = (int)rows;
    return launch_mix_i8_few(c, s);
  }
  const int8_t* w = static_cast<const int8_t*>(m.wq);
  Args p{};
  p.bias = m.bias;
  p.out = static_cast<char*>(m.out);
  p.pitch = i8_pitch(m.K);
  p.M = m.M;
  p.P = m.P;
  p.floor = m.relu ? 0.f : -INFINITY;
  p.stream = streams((double)rows * m.M, m.maps ? m.P : m.M, m.out_dt, m.out, m.out, 64);
  if (m.maps) {
    p.a = x; p.ascale = xscale; p.I = (int)rows;
    p.b = w; p.bscale = m.wscale; p.J = m.M;
    return m.out_dt == kBF16 ? launch<kBF16, true>(p, s) : launch<kF32, true>(p, s);
  }
  p.a = w; p.ascale = m.wscale; p.I = m.M;
  p.b = x; p.bscale = xscale; p.J = (int)rows;
  return m.out_dt == kBF16 ? launch<kBF16, false>(p, s) : launch<kF32, false>(p, s);
}

}  // namespace bc
