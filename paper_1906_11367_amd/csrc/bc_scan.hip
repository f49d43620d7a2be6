// The gated scan on token sequences [N][T][C] (gfx950): h_t = a_t h_{t-1} +
// b_t for every channel, forward and backward (bc_scan.hpp has the algebra).
//
// Bound by memory: the forward reads two tensors and writes one, the backward
// reads three and writes two, with 10 to 40 operations per element.  A block
// takes a slab of channels (whole cache lines of every row) by a tile of steps: a
// lane holds a few channels of a few consecutive steps in registers, so every
// element is read once.  A step is bound by its launch: 8 x 1024 2.5 us, 512 x
// 4096 bf16 6 to 7.5 (29 MB at 4.4 TB/s).
// 8 x 4096 x 2048 bf16: forward 89 us (4.5 TB/s), backward 143 (4.7 TB/s); 1 x
// 65536 x 1024 bf16 forward 100 (4.0); 64 x 512 x 1024 fp32 82 and 122 (4.9, 5.5):
// a copy of 1 GiB reaches 5.2 here, a plain elementwise kernel 6.2.  No tensor is
// read or written twice (counted: 1.01 of the bytes); a tile's loads, arithmetic and
// carries follow one another, and other blocks fill the gaps but not all of them.
#include "bc_scan.hpp"
#include "bc_scan_chain.hpp"

namespace bc {
namespace {

using namespace scan;

// The division of a tile: lanes hold kV channels of kL consecutive steps;
// kGroups lanes side by side make a slab (128 bytes or more: whole cache lines of
// every row), kSlots runs of steps a tile.  W_: waves per SIMD to build for.
template <int V_, int G_, int NT_, int L_, int W_>
struct Cut {
  static constexpr int kV = V_, kGroups = G_, kThreads = NT_, kL = L_, kWavesPerSimd = W_;
  static constexpr int kSlab = kV * kGroups, kSlots = kThreads / kGroups, kTile = kSlots * kL, kWaves = kThreads / 64;
};
// Cut 0 is the chained tiles'.  A sequence of one tile takes the shortest cut
// that holds it: a tile of 128 steps for a sequence of 4 would leave all but a
// few lanes of the block idle (256 x 4 x 4096 bf16 forward: 31 us instead of 11).
// Measured on 2^26 elements (bf16) and 2^25 (fp32) in chained tiles, us, other
// tensors from call to call, for 256 and for 16 chains:
//   forward, bf16: 4 channels x 8 steps a lane in 256 threads 90, 105; in 512
//     threads 99, 100; 8 x 8 in 512 132, 125; 2 x 8 in 512 91, 110
//   backward, bf16: 2 x 8 in 512 threads 146, 160; in 256 142, 178; 4 x 4 in 512
//     175, 180; 2 x 4 in 512 163, 193
//   fp32, 4 x 4 in 512 threads on 64 channels: forward 82, 85, backward 121, 123;
//     on 32 channels 93, 86 and 130, 126; in 256 threads on 32 82, 88 and 118, 127
// Longer tiles cost registers (fewer waves), shorter ones more carries.
// A few long chains wait for their carries, one after the other: the forward cuts
// them into half as many tiles (`far`), us at 4, 8 and 16 chains of 2048, 1024 and
// 512 tiles: bf16 112 for 158, 109 for 118, 100 for 105; fp32, 4 chains of 1024,
// 85 for 104.  At 32 chains of 256 tiles both take 98, and 2 of 32 tiles take 9.1
// for 7.7; the backward with such tiles takes 182 for 161 (16 chains).
template <class... Xs> struct CutList {};
template <int DT> struct FwdCuts;   // the chained cuts, then the others' tiles in rising order
template <> struct FwdCuts<kBF16> {
  using chained = Cut<4, 16, 256, 8, 4>;   // 128 steps
  using far = Cut<4, 16, 512, 8, 4>;       // 256
  using list = CutList<Cut<4, 64, 64, 8, 4>, Cut<4, 16, 64, 8, 4>, Cut<4, 16, 128, 8, 4>, chained,
                       far>;   // 8, 32, 64, 128, 256
};
template <> struct FwdCuts<kF32> {
  using chained = Cut<4, 16, 512, 4, 4>;   // 128
  using far = Cut<4, 16, 512, 8, 4>;       // 256
  using list = CutList<Cut<4, 64, 64, 8, 4>, Cut<4, 8, 64, 4, 4>, Cut<4, 8, 128, 4, 4>, chained,
                       Cut<4, 8, 512, 4, 4>>;   // 8, 32, 64, 128, 256
};
template <int DT> struct BwdCuts;
template <> struct BwdCuts<kBF16> {
  using chained = Cut<2, 32, 512, 8, 4>;   // 128
  using far = chained;
  using list = CutList<Cut<2, 64, 64, 8, 4>, Cut<2, 32, 64, 8, 4>, Cut<2, 32, 128, 8, 4>, Cut<2, 32, 256, 8, 4>,
                       chained>;   // 8, 16, 32, 64, 128
};
template <> struct BwdCuts<kF32> {
  using chained = Cut<4, 16, 512, 4, 4>;   // 128
  using far = chained;
  using list = CutList<Cut<4, 64, 64, 4, 4>, Cut<4, 8, 64, 4, 4>, Cut<4, 8, 128, 4, 4>, chained,
                       Cut<4, 8, 512, 4, 4>>;   // 4, 32, 64, 128, 256
};
// States are kept every kScanSpan steps: before every tile of the chained backward
// and before no other step (a sequence of one tile starts from its first state).
static_assert(BwdCuts<kBF16>::chained::kTile == kScanSpan && BwdCuts<kF32>::chained::kTile == kScanSpan, "kept states");

// (A, B) of the runs of lower slots of this wave (identity for the first), and
// the inclusive pair.  Slots are kGroups lanes apart.
template <int V, int kGroups>
__device__ __forceinline__ void wave_prefix(const float (&A)[V], const float (&B)[V], int lane, float (&iA)[V],
                                            float (&iB)[V], float (&eA)[V], float (&eB)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) { iA[k] = A[k]; iB[k] = B[k]; }
#pragma unroll
  for (int d = kGroups; d < 64; d *= 2) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float pa = __shfl_up(iA[k], d), pb = __shfl_up(iB[k], d);
      if (lane >= d) {
        iB[k] = __fmaf_rn(iA[k], pb, iB[k]);
        iA[k] *= pa;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float pa = __shfl_up(iA[k], kGroups), pb = __shfl_up(iB[k], kGroups);
    eA[k] = lane < kGroups ? 1.f : pa;
    eB[k] = lane < kGroups ? 0.f : pb;
  }
}

// The same from the other end: the runs of higher slots.
template <int V, int kGroups>
__device__ __forceinline__ void wave_suffix(const float (&A)[V], const float (&B)[V], int lane, float (&iA)[V],
                                            float (&iB)[V], float (&eA)[V], float (&eB)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) { iA[k] = A[k]; iB[k] = B[k]; }
#pragma unroll
  for (int d = kGroups; d < 64; d *= 2) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float pa = __shfl_down(iA[k], d), pb = __shfl_down(iB[k], d);
      if (lane + d < 64) {
        iB[k] = __fmaf_rn(iA[k], pb, iB[k]);
        iA[k] *= pa;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float pa = __shfl_down(iA[k], kGroups), pb = __shfl_down(iB[k], kGroups);
    eA[k] = lane >= 64 - kGroups ? 1.f : pa;
    eB[k] = lane >= 64 - kGroups ? 0.f : pb;
  }
}

// Chained tiles, the published single-pass scan with decoupled look-back (Merrill and
// Garland, 2016) in groups.  Every tile has a block of its own, and the state before
// a tile comes from the tiles before it in one launch: each publishes its pair
// (A, B), and a block combines the pairs back to the start of its group of
// kGroupTiles with the state published there (by the last block of the group
// before).  A block waits only on lower places of its chain, drawn as blocks
// start, whose owners are running and wait on still lower ones: every wait ends;
// which pairs are combined, and in which order, depends on the tile alone, so
// results do not depend on the order in which blocks run.
// A word carries its own validity: an 8-byte store is seen whole, and the
// workspace is first filled with kEmpty, which no publisher writes.
constexpr int kGroupTiles = 16;
constexpr unsigned long long kEmpty = ~0ull;
constexpr long kTicketWords = 16;   // a cache line for each counter
// A bound on the polls (about a second), past which a block goes on with a NaN.
// It is reached only where another call writes this one's workspace meanwhile:
// the outputs are then worthless, but every wait ends, and no access leaves the
// tensors or the workspace (chain_has).
constexpr int kMaxPolls = 1 << 20;

__device__ __forceinline__ void publish(unsigned long long* at, float lo, float hi) {
  if (hi != hi) hi = __uint_as_float(0x7fc00000u);   // never kEmpty
  const unsigned long long w = (unsigned long long)__float_as_uint(hi) << 32 | __float_as_uint(lo);
  __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ unsigned long long peek(const unsigned long long* at) {
  return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float word_lo(unsigned long long w) { return __uint_as_float((unsigned)w); }
__device__ __forceinline__ float word_hi(unsigned long long w) { return __uint_as_float((unsigned)(w >> 32)); }

// The words of a group that the lanes of one channel read: word 0 is the state
// at the group's start, word 1 + i the pair of its tile i.  Each of the block's
// kThreads / kSlab lanes of a channel takes a few consecutive ones and returns
// their composition (A = 0 where the state itself is among them; the first
// group's is in its tile 0's pair).
template <class X>
struct Lookback {
  static constexpr int kParts = X::kThreads / X::kSlab, kPer = (kGroupTiles + kParts - 1) / kParts;

  // o: the tile's place in its chain; first: the chain's start; agg and pre:
  // this channel's words of the chain
  static __device__ __forceinline__ void read(int o, int part, float first, const unsigned long long* agg,
                                              const unsigned long long* pre, float& A, float& B) {
    const int base = o & ~(kGroupTiles - 1), n = o - base;
    unsigned long long w[kPer];
    A = 1.f;
    B = 0.f;
    for (int polls = 0;; ++polls) {
      bool ready = true;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int k = part * kPer + i;
        const unsigned long long* at = k == 0 ? pre + (long)(base / kGroupTiles) * X::kSlab
                                              : agg + (long)(base + k - 1) * X::kSlab;
        w[i] = (k == 0 ? base > 0 : k <= n) ? peek(at) : 0ull;
        ready &= w[i] != kEmpty;
      }
      if (ready) break;
      if (polls == kMaxPolls) {
        A = B = __uint_as_float(0x7fc00000u);
        return;
      }
      __builtin_amdgcn_s_sleep(1);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = part * kPer + i;
      if (k == 0) {
        A = 0.f;
        B = base > 0 ? word_lo(w[i]) : first;   // first: 0 but in tile 0
      } else if (k <= n) {
        B = __fmaf_rn(word_hi(w[i]), B, word_lo(w[i]));
        A *= word_hi(w[i]);
      }
    }
  }
};

// Fills the words of a chained call (the counters with them: they start at -1).
__global__ __launch_bounds__(256) void k_scan_clear(unsigned long long* ws, long words) {
  const long i = (((long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x) * 2;
  if (i + 1 < words) *reinterpret_cast<ulonglong2*>(ws + i) = make_ulonglong2(kEmpty, kEmpty);
  else if (i < words) ws[i] = kEmpty;
}

// This block's unit and its place in the unit's chain, a ticket drawn from the
// unit's own counter: one counter for all serialised the blocks (about 15 ns a
// draw; with 8192 tiles 115 us instead of 90).  false, for the whole block: a
// block past the end (the grid's last row), or no place of the chain.
__device__ __forceinline__ bool draw_ticket(unsigned long long* tickets, int units, int tiles, int& unit, int& place) {
  __shared__ int t;
  const long b = (long)blockIdx.y * gridDim.x + blockIdx.x;
  if (b >= (long)units * tiles) return false;
  unit = chain_unit(b, units);
  if (threadIdx.x == 0) t = (int)(atomicAdd(reinterpret_cast<unsigned*>(tickets + (long)unit * kTicketWords), 1u) + 1u);
  __syncthreads();
  place = t;
  return chain_has(place, tiles);
}

template <class X, int IN, int OUT, int FORM, bool kChain>
__global__ __launch_bounds__(X::kThreads, X::kWavesPerSimd) void k_scan_fwd(FwdArgs p) {
  constexpr int V = X::kV, L = X::kL, CW = X::kSlab, kGroups = X::kGroups, kWaves = X::kWaves, kTile = X::kTile;
  __shared__ float totA[kWaves][CW], totB[kWaves][CW], carry[CW], last[CW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = tid % kGroups, slot = tid / kGroups;
  static_assert(!kChain || X::kThreads % CW == 0, "a chained tile's carries: a lane or more for each channel");
  constexpr int kParts = kChain ? X::kThreads / CW : 1;
  __shared__ float lookA[kParts][CW], lookB[kParts][CW];
  int unit, place = 0;
  if constexpr (kChain) {
    if (!draw_ticket(p.tickets, p.N * p.slabs, p.tiles, unit, place)) return;
  } else {
    const long b = (long)blockIdx.y * gridDim.x + blockIdx.x;
    if (b >= (long)p.N * p.slabs) return;
    unit = (int)b;
  }
  const int n = unit / p.slabs, slab = unit % p.slabs;
  const int c0 = slab * CW + grp * V, avail = p.C - c0;   // <= 0: no channel here
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + c0) * kBytes<IN>;
  char* yp = p.y + ((long)n * p.T * p.C + c0) * kBytes<OUT>;
  const int S = (p.T + kScanSpan - 1) / kScanSpan;
  auto start = [&](int ch) {
    const int c = slab * CW + ch;
    return p.h0 && c < p.C ? p.h0[(size_t)n * p.C + c] : 0.f;
  };
  float first = 0.f;
  if constexpr (kChain) {
    if (tid < CW && place == 0) first = start(tid);
  } else {   // a slab may have more channels than the block has lanes
    for (int ch = tid; ch < CW; ch += X::kThreads) carry[ch] = start(ch);
  }
  const int tile = place;
  const int t0 = tile * kTile + slot * L;
  // every lane has all of its elements, or none of a step's (past a sequence's
  // end, past the channels), or a part of them (the last channels)
  const bool whole = (tile + 1) * kTile <= len && (slab + 1) * CW <= p.C;
  const bool vectors = p.C % V == 0 || (slab + 1) * CW <= p.C;
  Raw<kWords<IN, V>> g[L], x[L];
  if (whole) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      g[i] = load_wide<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>);
      x[i] = load_wide<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>);
    }
  } else if (vectors) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      g[i] = hold_gate<IN, FORM, V>();
      x[i] = Raw<kWords<IN, V>>{};
    }
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (t0 + i < len && avail > 0) {
        g[i] = load_wide<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>);
        x[i] = load_wide<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>);
      }
  } else {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool on = t0 + i < len;
      g[i] = on ? load_vec<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>, avail) : hold_gate<IN, FORM, V>();
      x[i] = load_vec<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>, on ? avail : 0);
    }
  }
  float a[L][V], b[L][V], A[V], B[V];
#pragma unroll
  for (int k = 0; k < V; ++k) { A[k] = 1.f; B[k] = 0.f; }
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float c;
      coefficients<IN, FORM>(elem<IN, V>(g[i], k), a[i][k], c);
      b[i][k] = input_share<FORM>(c, elem<IN, V>(x[i], k));
      A[k] *= a[i][k];
      B[k] = __fmaf_rn(a[i][k], B[k], b[i][k]);
    }
  float iA[V], iB[V], eA[V], eB[V];
  wave_prefix<V, kGroups>(A, B, lane, iA, iB, eA, eB);
  if (lane >= 64 - kGroups) {
#pragma unroll
    for (int k = 0; k < V; ++k) { totA[wave][grp * V + k] = iA[k]; totB[wave][grp * V + k] = iB[k]; }
  }
  __syncthreads();
  if constexpr (kChain) {
    using Look = Lookback<X>;
    const int ch = tid % CW, part = tid / CW;
    const long chain = (long)unit * p.tiles * CW + ch, groups = (long)unit * p.groups * CW + ch;
    float ta = 1.f, tz = 0.f, A, B;
    if (tid < CW) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        tz = __fmaf_rn(totA[w][ch], tz, totB[w][ch]);
        ta *= totA[w][ch];
      }
      // tile 0 publishes a state (A = 0): only it reads the chain's start, whose
      // memory the chain's end may be
      if (place == 0) publish(p.agg + chain, __fmaf_rn(ta, first, tz), 0.f);
      else publish(p.agg + chain + (long)tile * CW, tz, ta);
    }
    Look::read(tile, part, first, p.agg + chain, p.pre + groups, A, B);
    lookA[part][ch] = A;
    lookB[part][ch] = B;
    __syncthreads();
    if (tid < CW) {
      float v = B;   // part 0 starts from the state itself
#pragma unroll
      for (int i = 1; i < kParts; ++i) v = __fmaf_rn(lookA[i][ch], v, lookB[i][ch]);
      carry[ch] = v;
      v = __fmaf_rn(ta, v, tz);
      last[ch] = v;
      if (tile % kGroupTiles == kGroupTiles - 1 && tile + 1 < p.tiles)
        publish(p.pre + groups + (long)(tile / kGroupTiles + 1) * CW, v, 0.f);
    }
    __syncthreads();
  } else {
    for (int ch = tid; ch < CW; ch += X::kThreads) {
      float h = carry[ch];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) h = __fmaf_rn(totA[w][ch], h, totB[w][ch]);
      last[ch] = h;
    }
  }
  float h[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    h[k] = carry[grp * V + k];
    for (int w = 0; w < wave; ++w) h[k] = __fmaf_rn(totA[w][grp * V + k], h[k], totB[w][grp * V + k]);
    h[k] = __fmaf_rn(eA[k], h[k], eB[k]);
  }
  if (p.states && t0 % kScanSpan == 0 && t0 < p.T && avail > 0)
    store_vec<kF32, V>(reinterpret_cast<char*>(p.states + ((size_t)n * S + t0 / kScanSpan) * p.C + c0), avail, h);
#pragma unroll
  for (int i = 0; i < L; ++i) {
#pragma unroll
    for (int k = 0; k < V; ++k) h[k] = __fmaf_rn(a[i][k], h[k], b[i][k]);
    char* at = yp + (long)(t0 + i) * p.C * kBytes<OUT>;
    if (whole) store_wide<OUT, V>(at, h, p.stream);
    else if (t0 + i < len) store_vec<OUT, V>(at, avail, h);   // avail <= 0: nothing
    else if (t0 + i < p.T) store_zero<OUT, V>(at, avail);
  }
  if (kChain && place + 1 < p.tiles) return;
  __syncthreads();
  if (p.h_last)
    for (int ch = tid; ch < CW && slab * CW + ch < p.C; ch += X::kThreads)
      p.h_last[(size_t)n * p.C + slab * CW + ch] = last[ch];
}

template <class X, int IN, int OUT, int FORM, bool kChain>
__global__ __launch_bounds__(X::kThreads, X::kWavesPerSimd) void k_scan_bwd(BwdArgs p) {
  constexpr int V = X::kV, L = X::kL, CW = X::kSlab, kGroups = X::kGroups, kWaves = X::kWaves, kTile = X::kTile;
  __shared__ float totA[kWaves][CW], totB[kWaves][CW], totR[kWaves][CW], carry[CW], last[CW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = tid % kGroups, slot = tid / kGroups;
  static_assert(!kChain || X::kThreads % CW == 0, "a chained tile's carries: a lane or more for each channel");
  constexpr int kParts = kChain ? X::kThreads / CW : 1;
  __shared__ float lookA[kParts][CW], lookB[kParts][CW];
  int unit, place = 0;
  if constexpr (kChain) {
    if (!draw_ticket(p.tickets, p.N * p.slabs, p.tiles, unit, place)) return;
  } else {
    const long b = (long)blockIdx.y * gridDim.x + blockIdx.x;
    if (b >= (long)p.N * p.slabs) return;
    unit = (int)b;
  }
  const int n = unit / p.slabs, slab = unit % p.slabs;
  const int c0 = slab * CW + grp * V, avail = p.C - c0;
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* gy = p.gy + ((long)n * p.T * p.C + c0) * kBytes<IN>;
  char* ggate = p.ggate + ((long)n * p.gbs + c0) * kBytes<OUT>;
  char* gx = p.gx + ((long)n * p.gbs + c0) * kBytes<OUT>;
  const int S = (p.T + kScanSpan - 1) / kScanSpan;
  auto start = [&](int ch) {
    const int c = slab * CW + ch;
    return p.gh_last && c < p.C ? p.gh_last[(size_t)n * p.C + c] : 0.f;
  };
  float first = 0.f;
  if constexpr (kChain) {
    if (tid < CW && place == 0) first = start(tid);
  } else {   // a slab may have more channels than the block has lanes
    for (int ch = tid; ch < CW; ch += X::kThreads) carry[ch] = start(ch);
  }
  const int o = place, tile = p.tiles - 1 - o;   // the chain runs backwards in time
  const int t0 = tile * kTile + slot * L;
  const bool whole = (tile + 1) * kTile <= len && (slab + 1) * CW <= p.C;
  const bool vectors = p.C % V == 0 || (slab + 1) * CW <= p.C;
  Raw<kWords<IN, V>> g[L], x[L], d[L];
  Raw<V> st;   // the state before the tile, kept by the forward
  const char* sp = reinterpret_cast<const char*>(p.states + ((size_t)n * S + tile * kTile / kScanSpan) * p.C + c0);
  if (whole) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      g[i] = load_wide<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>);
      x[i] = load_wide<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>);
      d[i] = load_wide<IN, V>(gy + (long)(t0 + i) * p.C * kBytes<IN>);
    }
    st = load_wide<kF32, V>(sp);
  } else if (vectors) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      g[i] = hold_gate<IN, FORM, V>();
      x[i] = d[i] = Raw<kWords<IN, V>>{};
    }
    st = Raw<V>{};
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (t0 + i < len && avail > 0) {
        g[i] = load_wide<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>);
        x[i] = load_wide<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>);
        d[i] = load_wide<IN, V>(gy + (long)(t0 + i) * p.C * kBytes<IN>);
      }
    if (avail > 0) st = load_wide<kF32, V>(sp);
  } else {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool on = t0 + i < len;
      g[i] = on ? load_vec<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>, avail) : hold_gate<IN, FORM, V>();
      x[i] = load_vec<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>, on ? avail : 0);
      d[i] = load_vec<IN, V>(gy + (long)(t0 + i) * p.C * kBytes<IN>, on ? avail : 0);
    }
    st = load_vec<kF32, V>(sp, avail);
  }
  float a[L][V], c[L][V], A[V], B[V], R[V];
#pragma unroll
  for (int k = 0; k < V; ++k) { A[k] = 1.f; B[k] = 0.f; R[k] = 0.f; }
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      coefficients<IN, FORM>(elem<IN, V>(g[i], k), a[i][k], c[i][k]);
      A[k] *= a[i][k];
      B[k] = __fmaf_rn(a[i][k], B[k], input_share<FORM>(c[i][k], elem<IN, V>(x[i], k)));
    }
#pragma unroll
  for (int i = L - 1; i >= 0; --i)
#pragma unroll
    for (int k = 0; k < V; ++k) R[k] = a[i][k] * (elem<IN, V>(d[i], k) + R[k]);
  float iA[V], iB[V], fA[V], fB[V], sA[V], sB[V];
  wave_prefix<V, kGroups>(A, B, lane, iA, iB, fA, fB);   // f: runs before this one
  if (lane >= 64 - kGroups) {
#pragma unroll
    for (int k = 0; k < V; ++k) { totA[wave][grp * V + k] = iA[k]; totB[wave][grp * V + k] = iB[k]; }
  }
  wave_suffix<V, kGroups>(A, R, lane, iA, iB, sA, sB);   // s: runs after it
  if (lane < kGroups) {
#pragma unroll
    for (int k = 0; k < V; ++k) totR[wave][grp * V + k] = iB[k];
  }
  __syncthreads();
  if constexpr (kChain) {
    using Look = Lookback<X>;
    const int ch = tid % CW, part = tid / CW;
    const long chain = (long)unit * p.tiles * CW + ch, groups = (long)unit * p.groups * CW + ch;
    float ta = 1.f, tz = 0.f, A, B;
    if (tid < CW) {
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) {
        tz = __fmaf_rn(totA[w][ch], tz, totR[w][ch]);
        ta *= totA[w][ch];
      }
      // tile 0 publishes a state (A = 0): only it reads the chain's start, whose
      // memory the chain's end may be
      if (place == 0) publish(p.agg + chain, __fmaf_rn(ta, first, tz), 0.f);
      else publish(p.agg + chain + (long)o * CW, tz, ta);
    }
    Look::read(o, part, first, p.agg + chain, p.pre + groups, A, B);
    lookA[part][ch] = A;
    lookB[part][ch] = B;
    __syncthreads();
    if (tid < CW) {
      float v = B;   // part 0 starts from the state itself
#pragma unroll
      for (int i = 1; i < kParts; ++i) v = __fmaf_rn(lookA[i][ch], v, lookB[i][ch]);
      carry[ch] = v;
      v = __fmaf_rn(ta, v, tz);
      last[ch] = v;
      if (o % kGroupTiles == kGroupTiles - 1 && o + 1 < p.tiles)
        publish(p.pre + groups + (long)(o / kGroupTiles + 1) * CW, v, 0.f);
    }
    __syncthreads();
  } else {
    for (int ch = tid; ch < CW; ch += X::kThreads) {
      float r = carry[ch];
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) r = __fmaf_rn(totA[w][ch], r, totR[w][ch]);
      last[ch] = r;
    }
  }
  float h[L][V], r[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int ch = grp * V + k;
    float hk = elem<kF32, V>(st, k);
    for (int w = 0; w < wave; ++w) hk = __fmaf_rn(totA[w][ch], hk, totB[w][ch]);
    h[0][k] = __fmaf_rn(fA[k], hk, fB[k]);
    float rk = carry[ch];
    for (int w = kWaves - 1; w > wave; --w) rk = __fmaf_rn(totA[w][ch], rk, totR[w][ch]);
    r[k] = __fmaf_rn(sA[k], rk, sB[k]);
  }
#pragma unroll
  for (int i = 0; i + 1 < L; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k)
      h[i + 1][k] = __fmaf_rn(a[i][k], h[i][k], input_share<FORM>(c[i][k], elem<IN, V>(x[i], k)));
#pragma unroll
  for (int i = L - 1; i >= 0; --i) {
    float og[V], ox[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float delta = elem<IN, V>(d[i], k) + r[k];
      if constexpr (FORM == kValue) {
        og[k] = delta * h[i][k];
        ox[k] = delta;
      } else {
        ox[k] = delta * c[i][k];
        og[k] = ox[k] * a[i][k] * (h[i][k] - elem<IN, V>(x[i], k));
      }
      r[k] = a[i][k] * delta;
    }
    char *gat = ggate + (long)(t0 + i) * p.grs * kBytes<OUT>, *xat = gx + (long)(t0 + i) * p.grs * kBytes<OUT>;
    if (whole) {
      store_wide<OUT, V>(gat, og, p.stream);
      store_wide<OUT, V>(xat, ox, p.stream);
    } else if (t0 + i < len) {
      store_vec<OUT, V>(gat, avail, og);
      store_vec<OUT, V>(xat, avail, ox);
    } else if (t0 + i < p.T) {
      store_zero<OUT, V>(gat, avail);
      store_zero<OUT, V>(xat, avail);
    }
  }
  if (kChain && place + 1 < p.tiles) return;
  __syncthreads();
  if (p.gh0)
    for (int ch = tid; ch < CW && slab * CW + ch < p.C; ch += X::kThreads)
      p.gh0[(size_t)n * p.C + slab * CW + ch] = last[ch];
}

// One token for N sequences: state rows from one pool to another (or in place).
// One lane per channel and row: a call is latency, or 3 e + 8 bytes an element.
template <int IN, int FORM>
__global__ __launch_bounds__(256) void k_scan_step(const char* gate, const char* x, long rs, const float* state,
                                                   float* state_out, const int* slots, char* y, int N, int C, int S,
                                                   int groups) {
  constexpr int V = 16 / kBytes<IN>;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const int n = (int)(i / groups), c0 = (int)(i % groups) * V;
  if (n >= N) return;
  const int avail = C - c0;
  const int s = slots ? slots[n] : n;
  const bool live = s >= 0 && s < S;
  float h[V];
#pragma unroll
  for (int k = 0; k < V; ++k) h[k] = 0.f;
  if (live) {
    const char *gp = gate + ((long)n * rs + c0) * kBytes<IN>, *xp = x + ((long)n * rs + c0) * kBytes<IN>;
    const char* sp = reinterpret_cast<const char*>(state + (size_t)s * C + c0);
    Raw<kWords<IN, V>> g, xv;
    Raw<V> st;
    if (C % V == 0) {
      g = load_wide<IN, V>(gp);
      xv = load_wide<IN, V>(xp);
      st = load_wide<kF32, V>(sp);
    } else {
      g = load_vec<IN, V>(gp, avail);
      xv = load_vec<IN, V>(xp, avail);
      st = load_vec<kF32, V>(sp, avail);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float a, c;
      coefficients<IN, FORM>(elem<IN, V>(g, k), a, c);
      h[k] = __fmaf_rn(a, elem<kF32, V>(st, k), input_share<FORM>(c, elem<IN, V>(xv, k)));
    }
    store_vec<kF32, V>(reinterpret_cast<char*>(state_out + (size_t)s * C + c0), avail, h);
  }
  store_vec<IN, V>(y + ((long)n * C + c0) * kBytes<IN>, avail, h);
}

// How a call on token sequences is divided, and its workspace: the chains'
// counters, a word per channel and tile, and one per channel and group.
struct Plan { int slab, tiles; long units, words; };   // words > 0: chained

template <class X>
Plan plan_of(int N, int T, int C) {
  Plan q{};
  q.slab = X::kSlab;
  q.tiles = (T + X::kTile - 1) / X::kTile;
  q.units = (long)N * ((C + X::kSlab - 1) / X::kSlab);
  const int groups = (q.tiles + kGroupTiles - 1) / kGroupTiles;
  if (q.tiles > 1) q.words = q.units * (kTicketWords + q.slab * ((long)q.tiles + groups));
  return q;
}

// Calls f with the cut of N x C sequences of T steps and whether its tiles are
// chained: the first of the list that holds the steps, or one of the chained.
template <class Cuts, class F, class X, class... Xs>
auto with_cut(int N, int T, int C, F f, CutList<X, Xs...>) {
  using Chained = typename Cuts::chained;
  using Far = typename Cuts::far;
  if (T <= X::kTile) return f(X{}, std::false_type{});
  if constexpr (sizeof...(Xs) > 0) {
    return with_cut<Cuts>(N, T, C, f, CutList<Xs...>{});
  } else {
    static_assert(X::kTile >= Chained::kTile, "more steps than the list holds: two tiles or more");
    const Plan q = plan_of<Chained>(N, T, C);
    if (q.tiles >= 128 && q.tiles >= 16 * q.units) return f(Far{}, std::true_type{});
    return f(Chained{}, std::true_type{});
  }
}
template <class Cuts, class F>
auto with_cut(int N, int T, int C, F f) { return with_cut<Cuts>(N, T, C, f, typename Cuts::list{}); }

// The workspace's words: the chained cut's where the far one, with half of them,
// is taken too, so that a workspace for longer sequences serves shorter ones.
template <class Cuts>
size_t words_of(int N, int T, int C) {
  return (size_t)with_cut<Cuts>(N, T, C, [&](auto, auto chained) {
    return decltype(chained)::value ? plan_of<typename Cuts::chained>(N, T, C).words : 0;
  });
}

// Launches the kernel of a cut; a chained one after a fill of its words.  Blocks
// past a grid's end return.
template <class X, bool kChain, class Args, class Kernel>
hipError_t launch_cut(Args& p, Kernel kernel, void* ws, hipStream_t s) {
  const Plan q = plan_of<X>(p.N, p.T, p.C);
  p.slabs = (int)(q.units / p.N);
  p.tiles = q.tiles;
  p.groups = (q.tiles + kGroupTiles - 1) / kGroupTiles;
  if constexpr (kChain) {
    unsigned long long* w = static_cast<unsigned long long*>(ws);
    p.tickets = w;
    p.agg = w + q.units * kTicketWords;
    p.pre = p.agg + q.units * q.tiles * q.slab;
    const Grid c = grid_of(clear_blocks(q.words));
    hipLaunchKernelGGL(k_scan_clear, dim3(c.x, c.y), dim3(256), 0, s, w, q.words);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const Grid g = grid_of(q.units * q.tiles);
  hipLaunchKernelGGL(kernel, dim3(g.x, g.y), dim3(X::kThreads), 0, s, p);
  return hipGetLastError();
}

template <int IN, int OUT, int FORM>
hipError_t fwd_form(FwdArgs& p, void* ws, hipStream_t s) {
  return with_cut<FwdCuts<IN>>(p.N, p.T, p.C, [&](auto x, auto chained) {
    using X = decltype(x);
    constexpr bool kChain = decltype(chained)::value;
    return launch_cut<X, kChain>(p, k_scan_fwd<X, IN, OUT, FORM, kChain>, ws, s);
  });
}

template <int IN, int OUT, int FORM>
hipError_t bwd_form(BwdArgs& p, void* ws, hipStream_t s) {
  return with_cut<BwdCuts<IN>>(p.N, p.T, p.C, [&](auto x, auto chained) {
    using X = decltype(x);
    constexpr bool kChain = decltype(chained)::value;
    return launch_cut<X, kChain>(p, k_scan_bwd<X, IN, OUT, FORM, kChain>, ws, s);
  });
}

template <int IN, int OUT>
hipError_t fwd_tokens(FwdArgs& p, int form, void* ws, hipStream_t s) {
  return form == kLogit ? fwd_form<IN, OUT, kLogit>(p, ws, s) : fwd_form<IN, OUT, kValue>(p, ws, s);
}

template <int IN, int OUT>
hipError_t bwd_tokens(BwdArgs& p, int form, void* ws, hipStream_t s) {
  return form == kLogit ? bwd_form<IN, OUT, kLogit>(p, ws, s) : bwd_form<IN, OUT, kValue>(p, ws, s);
}

}  // namespace

size_t scan_workspace_bytes(bool bwd, int N, int T, int C, int in_dt, bool maps) {
  if (maps) return 0;
  if (in_dt == kBF16) return 8 * (bwd ? words_of<BwdCuts<kBF16>>(N, T, C) : words_of<FwdCuts<kBF16>>(N, T, C));
  return 8 * (bwd ? words_of<BwdCuts<kF32>>(N, T, C) : words_of<FwdCuts<kF32>>(N, T, C));
}

hipError_t launch_scan_fwd(const ScanFwd& f, hipStream_t s) {
  FwdArgs p{};
  p.gate = static_cast<const char*>(f.gate);
  p.x = static_cast<const char*>(f.x);
  p.bs = f.bs;
  p.rs = f.rs;
  p.h0 = f.h0;
  p.lengths = f.lengths;
  p.y = static_cast<char*>(f.y);
  p.h_last = f.h_last;
  p.states = f.states;
  p.N = f.N;
  p.T = f.T;
  p.C = f.C;
  p.stream = streams((double)f.N * f.T * f.C, f.maps ? f.T : f.C, f.out_dt, f.y, f.y, f.maps ? 16 : 64);
  if (f.maps) return launch_scan_fwd_maps(p, f.in_dt, f.out_dt, f.form, s);
  if (f.in_dt == kBF16) return fwd_tokens<kBF16, kBF16>(p, f.form, f.ws, s);
  return f.out_dt == kBF16 ? fwd_tokens<kF32, kBF16>(p, f.form, f.ws, s) : fwd_tokens<kF32, kF32>(p, f.form, f.ws, s);
}

hipError_t launch_scan_bwd(const ScanBwd& f, hipStream_t s) {
  BwdArgs p{};
  p.gate = static_cast<const char*>(f.gate);
  p.x = static_cast<const char*>(f.x);
  p.bs = f.bs;
  p.rs = f.rs;
  p.states = f.states;
  p.lengths = f.lengths;
  p.gy = static_cast<const char*>(f.gy);
  p.gh_last = f.gh_last;
  p.ggate = static_cast<char*>(f.ggate);
  p.gx = static_cast<char*>(f.gx);
  p.gbs = f.gbs;
  p.grs = f.grs;
  p.gh0 = f.gh0;
  p.N = f.N;
  p.T = f.T;
  p.C = f.C;
  p.stream = streams((double)f.N * f.T * f.C, f.grs, f.out_dt, f.ggate, f.gx, f.maps ? 16 : 64) && f.gbs % (f.maps ? 8 : 32) == 0;
  if (f.maps) return launch_scan_bwd_maps(p, f.in_dt, f.out_dt, f.form, s);
  if (f.in_dt == kBF16) return bwd_tokens<kBF16, kBF16>(p, f.form, f.ws, s);
  return f.out_dt == kBF16 ? bwd_tokens<kF32, kBF16>(p, f.form, f.ws, s) : bwd_tokens<kF32, kF32>(p, f.form, f.ws, s);
}

hipError_t launch_scan_step(const void* gate, const void* x, long rs, int dt, const float* state, float* state_out,
                            const int* slots, void* y, int N, int C, int S, int form, hipStream_t s) {
  const int V = dt == kBF16 ? 8 : 4, groups = (C + V - 1) / V;
  const dim3 grid((unsigned)(((long)N * groups + 255) / 256));
  const char *g = static_cast<const char*>(gate), *xp = static_cast<const char*>(x);
  char* yp = static_cast<char*>(y);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, g, xp, rs, state, state_out, slots, yp, N, C, S, groups);
  };
  if (dt == kBF16) {
    if (form == kLogit) go(k_scan_step<kBF16, kLogit>);
    else go(k_scan_step<kBF16, kValue>);
  } else {
    if (form == kLogit) go(k_scan_step<kF32, kLogit>);
    else go(k_scan_step<kF32, kValue>);
  }
  return hipGetLastError();
}

}  // namespace bc
