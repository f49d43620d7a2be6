// The gated scan on token sequences [N][T][C] (gfx950): h_t = a_t h_{t-1} +
// b_t for every channel, forward and backward (bc_scan.hpp has the algebra).
//
// Bound by memory: the forward reads two tensors and writes one, the backward
// reads three and writes two, with 10 to 40 operations per element.  A block
// takes a slab of 128 bytes of channels (whole cache lines of every row) and
// walks tiles of kSlots * L steps: a lane holds 16 bytes of channels for L
// consecutive steps in registers, so every element is read once.
#include "bc_scan.hpp"

namespace bc {
namespace {

using namespace scan;

constexpr int kThreads = 256;
constexpr int kGroups = 8;                    // lanes across a slab
constexpr int kSlots = kThreads / kGroups;    // runs of steps in a tile
constexpr int kWaves = kThreads / 64;
template <int DT> constexpr int kV = 16 / kBytes<DT>;       // channels per lane
template <int DT> constexpr int kSlab = kGroups * kV<DT>;   // channels per block
constexpr int kFwdL = 8, kBwdL = 4;
constexpr int kFwdTile = kSlots * kFwdL, kBwdTile = kSlots * kBwdL;
// A state is kept every kScanSpan steps: where each backward tile starts.
static_assert(kBwdTile == kScanSpan && kFwdTile % kScanSpan == 0, "states at the backward's tiles");

// (A, B) of the runs of lower slots of this wave (identity for the first), and
// the inclusive pair.  Slots are kGroups lanes apart.
template <int V>
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
template <int V>
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

template <int IN, int OUT, int FORM>
__global__ __launch_bounds__(kThreads) void k_scan_fwd(FwdArgs p) {
  constexpr int V = kV<IN>, L = kFwdL, CW = kSlab<IN>;
  __shared__ float totA[2][kWaves][CW], totB[2][kWaves][CW], carry[2][CW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = tid % kGroups, slot = tid / kGroups;
  const int n = blockIdx.x / p.slabs, slab = blockIdx.x % p.slabs;
  const int c0 = slab * CW + grp * V, avail = p.C - c0;   // <= 0: no channel here
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + c0) * kBytes<IN>;
  char* yp = p.y + ((long)n * p.T * p.C + c0) * kBytes<OUT>;
  const int S = (p.T + kScanSpan - 1) / kScanSpan;
  if (tid < CW) {
    const int c = slab * CW + tid;
    carry[0][tid] = p.h0 && c < p.C ? p.h0[(size_t)n * p.C + c] : 0.f;
  }
  int q = 0;
  for (int tile = 0; tile < p.tiles; ++tile, q ^= 1) {
    const int t0 = tile * kFwdTile + slot * L;
    Raw<kWords<IN, V>> g[L], x[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int have = t0 + i < len ? avail : 0;
      g[i] = load_vec<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>, have);
      x[i] = load_vec<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>, have);
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
        if (t0 + i >= len) { a[i][k] = 1.f; b[i][k] = 0.f; }
        A[k] *= a[i][k];
        B[k] = __fmaf_rn(a[i][k], B[k], b[i][k]);
      }
    float iA[V], iB[V], eA[V], eB[V];
    wave_prefix<V>(A, B, lane, iA, iB, eA, eB);
    if (lane >= 64 - kGroups) {
#pragma unroll
      for (int k = 0; k < V; ++k) { totA[q][wave][grp * V + k] = iA[k]; totB[q][wave][grp * V + k] = iB[k]; }
    }
    __syncthreads();
    if (tid < CW) {
      float h = carry[q][tid];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) h = __fmaf_rn(totA[q][w][tid], h, totB[q][w][tid]);
      carry[q ^ 1][tid] = h;
    }
    float h[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      h[k] = carry[q][grp * V + k];
      for (int w = 0; w < wave; ++w) h[k] = __fmaf_rn(totA[q][w][grp * V + k], h[k], totB[q][w][grp * V + k]);
      h[k] = __fmaf_rn(eA[k], h[k], eB[k]);
    }
    if (p.states && t0 % kScanSpan == 0 && t0 < p.T && avail > 0)
      store_vec<kF32, V>(reinterpret_cast<char*>(p.states + ((size_t)n * S + t0 / kScanSpan) * p.C + c0), avail, h);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (t0 + i >= p.T) break;
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        h[k] = __fmaf_rn(a[i][k], h[k], b[i][k]);
        o[k] = t0 + i < len ? h[k] : 0.f;
      }
      store_vec<OUT, V>(yp + (long)(t0 + i) * p.C * kBytes<OUT>, avail, o);
    }
  }
  __syncthreads();
  if (p.h_last && tid < CW && slab * CW + tid < p.C) p.h_last[(size_t)n * p.C + slab * CW + tid] = carry[q][tid];
}

template <int IN, int OUT, int FORM>
__global__ __launch_bounds__(kThreads) void k_scan_bwd(BwdArgs p) {
  constexpr int V = kV<IN>, L = kBwdL, CW = kSlab<IN>;
  __shared__ float totA[2][kWaves][CW], totB[2][kWaves][CW], totR[2][kWaves][CW], carry[2][CW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = tid % kGroups, slot = tid / kGroups;
  const int n = blockIdx.x / p.slabs, slab = blockIdx.x % p.slabs;
  const int c0 = slab * CW + grp * V, avail = p.C - c0;
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + c0) * kBytes<IN>;
  const char* gy = p.gy + ((long)n * p.T * p.C + c0) * kBytes<IN>;
  char* ggate = p.ggate + ((long)n * p.gbs + c0) * kBytes<OUT>;
  char* gx = p.gx + ((long)n * p.gbs + c0) * kBytes<OUT>;
  if (tid < CW) {
    const int c = slab * CW + tid;
    carry[0][tid] = p.gh_last && c < p.C ? p.gh_last[(size_t)n * p.C + c] : 0.f;
  }
  int q = 0;
  for (int tile = p.tiles - 1; tile >= 0; --tile, q ^= 1) {
    const int t0 = tile * kBwdTile + slot * L;
    Raw<kWords<IN, V>> g[L], x[L], d[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int have = t0 + i < len ? avail : 0;
      g[i] = load_vec<IN, V>(gate + (long)(t0 + i) * p.rs * kBytes<IN>, have);
      x[i] = load_vec<IN, V>(xp + (long)(t0 + i) * p.rs * kBytes<IN>, have);
      d[i] = load_vec<IN, V>(gy + (long)(t0 + i) * p.C * kBytes<IN>, have);
    }
    // the state before the tile, kept by the forward
    const Raw<V> st = load_vec<kF32, V>(
        reinterpret_cast<const char*>(p.states + ((size_t)n * p.tiles + tile) * p.C + c0), avail);
    float a[L][V], c[L][V], A[V], B[V], R[V];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; B[k] = 0.f; R[k] = 0.f; }
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        coefficients<IN, FORM>(elem<IN, V>(g[i], k), a[i][k], c[i][k]);
        if (t0 + i >= len) { a[i][k] = 1.f; c[i][k] = 0.f; }   // x and grad_y read as zero there
        A[k] *= a[i][k];
        B[k] = __fmaf_rn(a[i][k], B[k], input_share<FORM>(c[i][k], elem<IN, V>(x[i], k)));
      }
#pragma unroll
    for (int i = L - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < V; ++k) R[k] = a[i][k] * (elem<IN, V>(d[i], k) + R[k]);
    float iA[V], iB[V], fA[V], fB[V], sA[V], sB[V];
    wave_prefix<V>(A, B, lane, iA, iB, fA, fB);   // f: runs before this one
    if (lane >= 64 - kGroups) {
#pragma unroll
      for (int k = 0; k < V; ++k) { totA[q][wave][grp * V + k] = iA[k]; totB[q][wave][grp * V + k] = iB[k]; }
    }
    wave_suffix<V>(A, R, lane, iA, iB, sA, sB);   // s: runs after it
    if (lane < kGroups) {
#pragma unroll
      for (int k = 0; k < V; ++k) totR[q][wave][grp * V + k] = iB[k];
    }
    __syncthreads();
    if (tid < CW) {
      float r = carry[q][tid];
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) r = __fmaf_rn(totA[q][w][tid], r, totR[q][w][tid]);
      carry[q ^ 1][tid] = r;
    }
    float h[L][V], r[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int ch = grp * V + k;
      float hk = elem<kF32, V>(st, k);
      for (int w = 0; w < wave; ++w) hk = __fmaf_rn(totA[q][w][ch], hk, totB[q][w][ch]);
      h[0][k] = __fmaf_rn(fA[k], hk, fB[k]);
      float rk = carry[q][ch];
      for (int w = kWaves - 1; w > wave; --w) rk = __fmaf_rn(totA[q][w][ch], rk, totR[q][w][ch]);
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
        if (t0 + i >= len) og[k] = ox[k] = 0.f;
      }
      if (t0 + i < p.T) {
        store_vec<OUT, V>(ggate + (long)(t0 + i) * p.grs * kBytes<OUT>, avail, og);
        store_vec<OUT, V>(gx + (long)(t0 + i) * p.grs * kBytes<OUT>, avail, ox);
      }
    }
  }
  __syncthreads();
  if (p.gh0 && tid < CW && slab * CW + tid < p.C) p.gh0[(size_t)n * p.C + slab * CW + tid] = carry[q][tid];
}

// One token for N sequences: state rows from one pool to another (or in place).
// One lane per channel and row: a call is latency, or 3 e + 8 bytes an element.
template <int IN, int FORM>
__global__ __launch_bounds__(256) void k_scan_step(const char* gate, const char* x, long rs, const float* state,
                                                   float* state_out, const int* slots, char* y, int N, int C, int S,
                                                   int groups) {
  constexpr int V = kV<IN>;
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
    const auto g = load_vec<IN, V>(gate + ((long)n * rs + c0) * kBytes<IN>, avail);
    const auto xv = load_vec<IN, V>(x + ((long)n * rs + c0) * kBytes<IN>, avail);
    const auto st = load_vec<kF32, V>(reinterpret_cast<const char*>(state + (size_t)s * C + c0), avail);
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

template <int IN, int OUT>
hipError_t fwd_tokens(FwdArgs& p, int form, hipStream_t s) {
  p.slabs = (p.C + kSlab<IN> - 1) / kSlab<IN>;
  p.tiles = (p.T + kFwdTile - 1) / kFwdTile;
  const dim3 grid((unsigned)(p.N * p.slabs));
  if (form == kLogit) hipLaunchKernelGGL((k_scan_fwd<IN, OUT, kLogit>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((k_scan_fwd<IN, OUT, kValue>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <int IN, int OUT>
hipError_t bwd_tokens(BwdArgs& p, int form, hipStream_t s) {
  p.slabs = (p.C + kSlab<IN> - 1) / kSlab<IN>;
  p.tiles = (p.T + kBwdTile - 1) / kBwdTile;
  const dim3 grid((unsigned)(p.N * p.slabs));
  if (form == kLogit) hipLaunchKernelGGL((k_scan_bwd<IN, OUT, kLogit>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((k_scan_bwd<IN, OUT, kValue>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

size_t scan_workspace_bytes(bool, int, int, int, int, bool) { return 0; }

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
  if (f.maps) return launch_scan_fwd_maps(p, f.in_dt, f.out_dt, f.form, s);
  if (f.in_dt == kBF16) return fwd_tokens<kBF16, kBF16>(p, f.form, s);
  return f.out_dt == kBF16 ? fwd_tokens<kF32, kBF16>(p, f.form, s) : fwd_tokens<kF32, kF32>(p, f.form, s);
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
  if (f.maps) return launch_scan_bwd_maps(p, f.in_dt, f.out_dt, f.form, s);
  if (f.in_dt == kBF16) return bwd_tokens<kBF16, kBF16>(p, f.form, s);
  return f.out_dt == kBF16 ? bwd_tokens<kF32, kBF16>(p, f.form, s) : bwd_tokens<kF32, kF32>(p, f.form, s);
}

hipError_t launch_scan_step(const void* gate, const void* x, long rs, int dt, const float* state, float* state_out,
                            const int* slots, void* y, int N, int C, int S, int form, hipStream_t s) {
  const int V = dt == kBF16 ? kV<kBF16> : kV<kF32>, groups = (C + V - 1) / V;
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
