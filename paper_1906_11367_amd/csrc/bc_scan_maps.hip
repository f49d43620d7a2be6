// The gated scan on maps [N][C][T] (gfx950): every row is one sequence, time
// contiguous, as the 1x1 mix writes its outputs (bc_scan.hpp has the algebra).
//
// A wave takes 512 (bf16) or 256 (fp32) consecutive steps of a row at a time,
// 16 bytes to a lane, scans the lanes' pairs by lane moves and carries the
// state on.  W waves share a row, a segment each, where there are too few rows
// for a wave each.
// Bound by memory: 32 x 256 x 64 x 64 fp32 forward 80 us (5.0 TB/s), backward 124
// (5.4 TB/s), where a copy of 1 GiB reaches 5.2 and a plain elementwise kernel 6.2;
// a few long rows by one CU's loads each (24 of 65536 bf16: 18 us, 0.5 TB/s).
#include "bc_scan.hpp"

namespace bc {
namespace {

using namespace scan;

// Steps a lane (16 bytes: a wave's access is 1 KiB in one piece), and a wave's
// segment, at each of which a state is kept.
template <int DT> constexpr int kV = DT == kBF16 ? 8 : 4;
template <int DT> constexpr int kSeg = 64 * kV<DT>;
static_assert(kSeg<kBF16> % kScanSpanMaps == 0 && kSeg<kF32> % kScanSpanMaps == 0, "room for the states");

// Runs of lower lanes of a group of G lanes (lane: within the group).
template <int G>
__device__ __forceinline__ void lanes_prefix(float& A, float& B, int lane, float& eA, float& eB) {
#pragma unroll
  for (int d = 1; d < G; d *= 2) {
    const float pa = __shfl_up(A, d), pb = __shfl_up(B, d);
    if (lane >= d) {
      B = __fmaf_rn(A, pb, B);
      A *= pa;
    }
  }
  eA = __shfl_up(A, 1);
  eB = __shfl_up(B, 1);
  if (lane == 0) { eA = 1.f; eB = 0.f; }
}

// Runs of higher lanes.
template <int G>
__device__ __forceinline__ void lanes_suffix(float& A, float& B, int lane, float& eA, float& eB) {
#pragma unroll
  for (int d = 1; d < G; d *= 2) {
    const float pa = __shfl_down(A, d), pb = __shfl_down(B, d);
    if (lane + d < G) {
      B = __fmaf_rn(A, pb, B);
      A *= pa;
    }
  }
  eA = __shfl_down(A, 1);
  eB = __shfl_down(B, 1);
  if (lane == G - 1) { eA = 1.f; eB = 0.f; }
}

// W waves to a row; blocks of kRows rows.
template <int W> constexpr int kRows = W >= 4 ? 1 : 4 / W;

template <int IN, int OUT, int FORM, int W>
__global__ __launch_bounds__(64 * W * kRows<W>) void k_scan_fwd_maps(FwdArgs p) {
  constexpr int V = kV<IN>, Seg = kSeg<IN>;
  __shared__ float tot[2][W][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
  const long row = (long)blockIdx.x * kRows<W> + wave / W;
  if (row >= (long)p.N * p.C) return;   // W > 1: the whole block has one row
  const int n = (int)(row / p.C), c = (int)(row % p.C);
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + (long)c * p.rs) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + (long)c * p.rs) * kBytes<IN>;
  char* yp = p.y + row * p.T * kBytes<OUT>;
  const int S = (p.T + Seg - 1) / Seg;
  float carry = p.h0 ? p.h0[row] : 0.f;
  int q = 0;
  Raw<kWords<IN, V>> g, x;
  auto load = [&](int seg) {
    const int t = seg * Seg + lane * V;
    if ((seg + 1) * Seg <= len) {   // for every lane
      g = load_wide<IN, V>(gate + (long)t * kBytes<IN>);
      x = load_wide<IN, V>(xp + (long)t * kBytes<IN>);
    } else {
      g = load_vec<IN, V>(gate + (long)t * kBytes<IN>, len - t);
      x = load_vec<IN, V>(xp + (long)t * kBytes<IN>, len - t);
    }
  };
  load(w);
  for (int s0 = 0; s0 < S; s0 += W, q ^= 1) {
    const int t0 = (s0 + w) * Seg + lane * V;
    const bool whole = (s0 + w + 1) * Seg <= len;
    float a[V], b[V], A = 1.f, B = 0.f, eA, eB;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float cx;
      coefficients<IN, FORM>(elem<IN, V>(g, k), a[k], cx);
      b[k] = input_share<FORM>(cx, elem<IN, V>(x, k));
      if (t0 + k >= len) { a[k] = 1.f; b[k] = 0.f; }
      A *= a[k];
      B = __fmaf_rn(a[k], B, b[k]);
    }
    if (s0 + W < S) load(s0 + W + w);   // on its way meanwhile
    lanes_prefix<64>(A, B, lane, eA, eB);
    float hw = carry;   // the state before this wave's segment
    if constexpr (W == 1) {
      carry = __fmaf_rn(__shfl(A, 63), carry, __shfl(B, 63));
    } else {
      if (lane == 63) { tot[q][w][0] = A; tot[q][w][1] = B; }
      __syncthreads();
      for (int i = 0; i < W; ++i) {
        if (i == w) hw = carry;
        carry = __fmaf_rn(tot[q][i][0], carry, tot[q][i][1]);
      }
    }
    if (p.states && lane == 0 && s0 + w < S) p.states[row * S + s0 + w] = hw;
    float h = __fmaf_rn(eA, hw, eB), o[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      h = __fmaf_rn(a[k], h, b[k]);
      o[k] = t0 + k < len ? h : 0.f;
    }
    if (whole) store_wide<OUT, V>(yp + (long)t0 * kBytes<OUT>, o, p.stream);
    else store_vec<OUT, V>(yp + (long)t0 * kBytes<OUT>, p.T - t0, o);
  }
  if (p.h_last && w == 0 && lane == 0) p.h_last[row] = carry;
}

template <int IN, int OUT, int FORM, int W>
__global__ __launch_bounds__(64 * W * kRows<W>) void k_scan_bwd_maps(BwdArgs p) {
  constexpr int V = kV<IN>, Seg = kSeg<IN>;
  __shared__ float tot[2][W][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
  const long row = (long)blockIdx.x * kRows<W> + wave / W;
  if (row >= (long)p.N * p.C) return;
  const int n = (int)(row / p.C), c = (int)(row % p.C);
  const int len = seq_len(p.lengths, n, p.T);
  const char* gate = p.gate + ((long)n * p.bs + (long)c * p.rs) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + (long)c * p.rs) * kBytes<IN>;
  const char* gy = p.gy + row * p.T * kBytes<IN>;
  char* ggate = p.ggate + ((long)n * p.gbs + (long)c * p.grs) * kBytes<OUT>;
  char* gx = p.gx + ((long)n * p.gbs + (long)c * p.grs) * kBytes<OUT>;
  const int S = (p.T + Seg - 1) / Seg;
  float carry = p.gh_last ? p.gh_last[row] : 0.f;
  int q = 0;
  struct Piece {
    Raw<kWords<IN, V>> g, x, d;
    float st;   // the state before the segment
  };
  auto load = [&](int seg) {
    const int t = seg * Seg + lane * V;
    Piece r;
    if ((seg + 1) * Seg <= len) {   // for every lane
      r.g = load_wide<IN, V>(gate + (long)t * kBytes<IN>);
      r.x = load_wide<IN, V>(xp + (long)t * kBytes<IN>);
      r.d = load_wide<IN, V>(gy + (long)t * kBytes<IN>);
    } else {
      r.g = load_vec<IN, V>(gate + (long)t * kBytes<IN>, len - t);
      r.x = load_vec<IN, V>(xp + (long)t * kBytes<IN>, len - t);
      r.d = load_vec<IN, V>(gy + (long)t * kBytes<IN>, len - t);
    }
    r.st = seg < S ? p.states[row * S + seg] : 0.f;
    return r;
  };
  const int top = (S - 1) / W * W;
  Piece next = load(top + w);
  for (int s0 = top; s0 >= 0; s0 -= W, q ^= 1) {
    const int t0 = (s0 + w) * Seg + lane * V;
    const bool whole = (s0 + w + 1) * Seg <= len;
    const Piece now = next;
    if (s0 > 0) next = load(s0 - W + w);   // on its way meanwhile
    const auto &g = now.g, &xr = now.x, &dr = now.d;
    const float st = now.st;
    float a[V], cx[V], h[V], A = 1.f, B = 0.f, R = 0.f, eA, eB, sA, sB;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      coefficients<IN, FORM>(elem<IN, V>(g, k), a[k], cx[k]);
      if (t0 + k >= len) { a[k] = 1.f; cx[k] = 0.f; }
      A *= a[k];
      B = __fmaf_rn(a[k], B, input_share<FORM>(cx[k], elem<IN, V>(xr, k)));
    }
#pragma unroll
    for (int k = V - 1; k >= 0; --k) R = a[k] * (elem<IN, V>(dr, k) + R);
    float fA = A, fB = B;
    lanes_prefix<64>(fA, fB, lane, eA, eB);
    lanes_suffix<64>(A, R, lane, sA, sB);
    float rw = carry;   // the gradient carried into this wave's segment from after it
    if constexpr (W == 1) {
      carry = __fmaf_rn(__shfl(A, 0), carry, __shfl(R, 0));
    } else {
      if (lane == 0) { tot[q][w][0] = A; tot[q][w][1] = R; }
      __syncthreads();
      for (int i = W - 1; i >= 0; --i) {
        if (i == w) rw = carry;
        carry = __fmaf_rn(tot[q][i][0], carry, tot[q][i][1]);
      }
    }
    h[0] = __fmaf_rn(eA, st, eB);
#pragma unroll
    for (int k = 0; k + 1 < V; ++k)
      h[k + 1] = __fmaf_rn(a[k], h[k], input_share<FORM>(cx[k], elem<IN, V>(xr, k)));
    float r = __fmaf_rn(sA, rw, sB), og[V], ox[V];
#pragma unroll
    for (int k = V - 1; k >= 0; --k) {
      const float delta = elem<IN, V>(dr, k) + r;
      if constexpr (FORM == kValue) {
        og[k] = delta * h[k];
        ox[k] = delta;
      } else {
        ox[k] = delta * cx[k];
        og[k] = ox[k] * a[k] * (h[k] - elem<IN, V>(xr, k));
      }
      r = a[k] * delta;
      if (t0 + k >= len) og[k] = ox[k] = 0.f;
    }
    if (whole) {
      store_wide<OUT, V>(ggate + (long)t0 * kBytes<OUT>, og, p.stream);
      store_wide<OUT, V>(gx + (long)t0 * kBytes<OUT>, ox, p.stream);
    } else {
      store_vec<OUT, V>(ggate + (long)t0 * kBytes<OUT>, p.T - t0, og);
      store_vec<OUT, V>(gx + (long)t0 * kBytes<OUT>, p.T - t0, ox);
    }
  }
  if (p.gh0 && w == 0 && lane == 0) p.gh0[row] = carry;
}

// Short rows: G lanes to a row, 64 / G rows to a wave, T <= G * V.
template <int IN, int OUT, int FORM, int G>
__global__ __launch_bounds__(256) void k_scan_fwd_short(FwdArgs p) {
  constexpr int V = kV<IN>;
  const int sub = threadIdx.x & (G - 1);
  const long row = (long)blockIdx.x * (256 / G) + threadIdx.x / G;
  const bool on = row < (long)p.N * p.C;   // all lanes of the wave take part in the lane moves
  const int n = on ? (int)(row / p.C) : 0, c = on ? (int)(row % p.C) : 0;
  const int len = on ? seq_len(p.lengths, n, p.T) : 0, t0 = sub * V;
  const char* gate = p.gate + ((long)n * p.bs + (long)c * p.rs + t0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + (long)c * p.rs + t0) * kBytes<IN>;
  Raw<kWords<IN, V>> g = {}, x = {};
  if (__any(t0 < len && t0 + V > len)) {
    g = load_vec<IN, V>(gate, len - t0);
    x = load_vec<IN, V>(xp, len - t0);
  } else if (t0 < len) {
    g = load_wide<IN, V>(gate);
    x = load_wide<IN, V>(xp);
  }
  float a[V], b[V], A = 1.f, B = 0.f, eA, eB, o[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float cx;
    coefficients<IN, FORM>(elem<IN, V>(g, k), a[k], cx);
    b[k] = input_share<FORM>(cx, elem<IN, V>(x, k));
    if (t0 + k >= len) { a[k] = 1.f; b[k] = 0.f; }
    A *= a[k];
    B = __fmaf_rn(a[k], B, b[k]);
  }
  lanes_prefix<G>(A, B, sub, eA, eB);
  const float first = on && p.h0 ? p.h0[row] : 0.f;
  float h = __fmaf_rn(eA, first, eB);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    h = __fmaf_rn(a[k], h, b[k]);
    o[k] = t0 + k < len ? h : 0.f;
  }
  if (!on) return;
  if (p.states && sub == 0) p.states[row] = first;
  store_vec<OUT, V>(p.y + (row * p.T + t0) * kBytes<OUT>, p.T - t0, o);
  if (p.h_last && sub == G - 1) p.h_last[row] = h;
}

template <int IN, int OUT, int FORM, int G>
__global__ __launch_bounds__(256) void k_scan_bwd_short(BwdArgs p) {
  constexpr int V = kV<IN>;
  const int sub = threadIdx.x & (G - 1);
  const long row = (long)blockIdx.x * (256 / G) + threadIdx.x / G;
  const bool on = row < (long)p.N * p.C;
  const int n = on ? (int)(row / p.C) : 0, c = on ? (int)(row % p.C) : 0;
  const int len = on ? seq_len(p.lengths, n, p.T) : 0, t0 = sub * V;
  const char* gate = p.gate + ((long)n * p.bs + (long)c * p.rs + t0) * kBytes<IN>;
  const char* xp = p.x + ((long)n * p.bs + (long)c * p.rs + t0) * kBytes<IN>;
  const char* gy = p.gy + ((on ? row : 0) * p.T + t0) * kBytes<IN>;
  Raw<kWords<IN, V>> g = {}, x = {}, d = {};
  if (__any(t0 < len && t0 + V > len)) {
    g = load_vec<IN, V>(gate, len - t0);
    x = load_vec<IN, V>(xp, len - t0);
    d = load_vec<IN, V>(gy, len - t0);
  } else if (t0 < len) {
    g = load_wide<IN, V>(gate);
    x = load_wide<IN, V>(xp);
    d = load_wide<IN, V>(gy);
  }
  float a[V], cx[V], h[V], A = 1.f, B = 0.f, R = 0.f, eA, eB, sA, sB, og[V], ox[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    coefficients<IN, FORM>(elem<IN, V>(g, k), a[k], cx[k]);
    if (t0 + k >= len) { a[k] = 1.f; cx[k] = 0.f; }
    A *= a[k];
    B = __fmaf_rn(a[k], B, input_share<FORM>(cx[k], elem<IN, V>(x, k)));
  }
#pragma unroll
  for (int k = V - 1; k >= 0; --k) R = a[k] * (elem<IN, V>(d, k) + R);
  float fA = A, fB = B;
  lanes_prefix<G>(fA, fB, sub, eA, eB);
  lanes_suffix<G>(A, R, sub, sA, sB);
  const float last = on && p.gh_last ? p.gh_last[row] : 0.f;
  h[0] = __fmaf_rn(eA, on ? p.states[row] : 0.f, eB);
#pragma unroll
  for (int k = 0; k + 1 < V; ++k) h[k + 1] = __fmaf_rn(a[k], h[k], input_share<FORM>(cx[k], elem<IN, V>(x, k)));
  float r = __fmaf_rn(sA, last, sB);
#pragma unroll
  for (int k = V - 1; k >= 0; --k) {
    const float delta = elem<IN, V>(d, k) + r;
    if constexpr (FORM == kValue) {
      og[k] = delta * h[k];
      ox[k] = delta;
    } else {
      ox[k] = delta * cx[k];
      og[k] = ox[k] * a[k] * (h[k] - elem<IN, V>(x, k));
    }
    r = a[k] * delta;
    if (t0 + k >= len) og[k] = ox[k] = 0.f;
  }
  if (!on) return;
  store_vec<OUT, V>(p.ggate + ((long)n * p.gbs + (long)c * p.grs + t0) * kBytes<OUT>, p.T - t0, og);
  store_vec<OUT, V>(p.gx + ((long)n * p.gbs + (long)c * p.grs + t0) * kBytes<OUT>, p.T - t0, ox);
  if (p.gh0 && sub == 0) p.gh0[row] = r;
}

// Waves to a row: as many as the row has segments for, until there are 4096
// waves in all (four for each SIMD).
int waves_per_row(int N, int C, int T, int seg) {
  const long rows = (long)N * C;
  const int segs = (T + seg - 1) / seg;
  int w = 1;
  while (w < 16 && w < segs && rows * w < 4096) w *= 4;
  return w;
}

template <int W, class Args, class Kernel>
hipError_t launch_rows(Kernel kernel, const Args& p, hipStream_t s) {
  const long rows = (long)p.N * p.C;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + kRows<W> - 1) / kRows<W>)), dim3(64 * W * kRows<W>), 0, s, p);
  return hipGetLastError();
}

template <int G, class Args, class Kernel>
hipError_t launch_short(Kernel kernel, const Args& p, hipStream_t s) {
  const long rows = (long)p.N * p.C;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 256 / G - 1) / (256 / G))), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <int IN, int OUT, int FORM>
hipError_t fwd_rows(const FwdArgs& p, hipStream_t s) {
  constexpr int V = kV<IN>;
  if (p.T <= V) return launch_short<1>(k_scan_fwd_short<IN, OUT, FORM, 1>, p, s);
  if (p.T <= 4 * V) return launch_short<4>(k_scan_fwd_short<IN, OUT, FORM, 4>, p, s);
  if (p.T <= 16 * V) return launch_short<16>(k_scan_fwd_short<IN, OUT, FORM, 16>, p, s);
  if (p.T <= 32 * V) return launch_short<32>(k_scan_fwd_short<IN, OUT, FORM, 32>, p, s);
  switch (waves_per_row(p.N, p.C, p.T, kSeg<IN>)) {
    case 1: return launch_rows<1>(k_scan_fwd_maps<IN, OUT, FORM, 1>, p, s);
    case 4: return launch_rows<4>(k_scan_fwd_maps<IN, OUT, FORM, 4>, p, s);
    default: return launch_rows<16>(k_scan_fwd_maps<IN, OUT, FORM, 16>, p, s);
  }
}

template <int IN, int OUT, int FORM>
hipError_t bwd_rows(const BwdArgs& p, hipStream_t s) {
  constexpr int V = kV<IN>;
  if (p.T <= V) return launch_short<1>(k_scan_bwd_short<IN, OUT, FORM, 1>, p, s);
  if (p.T <= 4 * V) return launch_short<4>(k_scan_bwd_short<IN, OUT, FORM, 4>, p, s);
  if (p.T <= 16 * V) return launch_short<16>(k_scan_bwd_short<IN, OUT, FORM, 16>, p, s);
  if (p.T <= 32 * V) return launch_short<32>(k_scan_bwd_short<IN, OUT, FORM, 32>, p, s);
  switch (waves_per_row(p.N, p.C, p.T, kSeg<IN>)) {
    case 1: return launch_rows<1>(k_scan_bwd_maps<IN, OUT, FORM, 1>, p, s);
    case 4: return launch_rows<4>(k_scan_bwd_maps<IN, OUT, FORM, 4>, p, s);
    default: return launch_rows<16>(k_scan_bwd_maps<IN, OUT, FORM, 16>, p, s);
  }
}

}  // namespace

hipError_t launch_scan_fwd_maps(const scan::FwdArgs& p, int in_dt, int out_dt, int form, hipStream_t s) {
  auto go = [&](auto f) {
    constexpr int F = decltype(f)::value;
    if (in_dt == kBF16) return fwd_rows<kBF16, kBF16, F>(p, s);
    return out_dt == kBF16 ? fwd_rows<kF32, kBF16, F>(p, s) : fwd_rows<kF32, kF32, F>(p, s);
  };
  return form == kLogit ? go(std::integral_constant<int, kLogit>{}) : go(std::integral_constant<int, kValue>{});
}

hipError_t launch_scan_bwd_maps(const scan::BwdArgs& p, int in_dt, int out_dt, int form, hipStream_t s) {
  auto go = [&](auto f) {
    constexpr int F = decltype(f)::value;
    if (in_dt == kBF16) return bwd_rows<kBF16, kBF16, F>(p, s);
    return out_dt == kBF16 ? bwd_rows<kF32, kBF16, F>(p, s) : bwd_rows<kF32, kF32, F>(p, s);
  };
  return form == kLogit ? go(std::integral_constant<int, kLogit>{}) : go(std::integral_constant<int, kValue>{});
}

}  // namespace bc
