// The walk of linear attention over a segment (bc_linattn.hpp), on MFMA.
//
// A block of four waves takes a segment of one sequence and head, chunk by
// chunk: q, k and v of a chunk go through LDS, each wave owns a quarter of the
// state's columns (v's), which stay in its registers as fp32 accumulators, and
// the chunk's scores, one 16 x 16 tile at a time, are shared through LDS.
//
// The matrix instruction (16 x 16 outputs) wants both operands by rows of the
// reduction, 4 or 8 consecutive per lane, and leaves 4 consecutive rows of its
// output with a lane; a reduction may run in any order that both operands
// share.  So the accumulators of S are an operand of q S as they are (the
// columns of q that a lane reads are the rows of S that it holds), and scores
// computed as k q^T are one of (scores) v; nothing is transposed but the rows
// of k and v, by the LDS read that does it (ds_read_b64_tr_b16).
//
// bf16: fp32 values that meet bf16 inputs in a product are split into sums of
// bf16 (each the rest of the one before), so that only the storage type rounds:
// scores and S into two (to 2^-17 of themselves; they make outputs of 2^-9), the
// decayed v that the state takes in into three (2^-25: the state is fp32).
// fp32: the fp32 matrix instruction.
#pragma once
#include "bc_linattn.hpp"

namespace bc {
namespace linattn {
namespace {

template <int DT> struct Traits;
template <> struct Traits<kBF16> {
  static constexpr int kChunk = 64, kGroup = 32;   // tokens of a chunk; reduction of one operand pair
  using Frag = bf16x8_t;
  using Elem = uint16_t;
};
template <> struct Traits<kF32> {
  static constexpr int kChunk = 32, kGroup = 16;
  using Frag = f32x4_t;
  using Elem = float;
};

__device__ __forceinline__ f32x4_t mma(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma(const f32x4_t& a, const f32x4_t& b, f32x4_t c) {
#pragma unroll
  for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
  return c;
}

// fp32 values as a sum of P operands.
template <int DT, int P> struct Split {
  typename Traits<DT>::Frag part[DT == kBF16 ? P : 1];
};
template <int P>
__device__ __forceinline__ Split<kBF16, P> split(const float (&x)[8]) {
  Split<kBF16, P> s;
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const __bf16 h = (__bf16)rest[e];
      s.part[p][e] = h;
      if (p + 1 < P) rest[e] -= (float)h;
    }
  }
  return s;
}
template <int P>
__device__ __forceinline__ Split<kF32, P> split(const float (&x)[4]) {
  Split<kF32, P> s;
#pragma unroll
  for (int e = 0; e < 4; ++e) s.part[0][e] = x[e];
  return s;
}
template <int DT, int P>
__device__ __forceinline__ f32x4_t mma(const Split<DT, P>& a, const typename Traits<DT>::Frag& b, f32x4_t c) {
#pragma unroll
  for (int p = (DT == kBF16 ? P : 1) - 1; p >= 0; --p) c = mma(a.part[p], b, c);
  return c;
}
template <int DT, int P>
__device__ __forceinline__ f32x4_t mma(const typename Traits<DT>::Frag& a, const Split<DT, P>& b, f32x4_t c) {
#pragma unroll
  for (int p = (DT == kBF16 ? P : 1) - 1; p >= 0; --p) c = mma(a, b.part[p], c);
  return c;
}

// A chunk's rows of one operand: from memory to registers, then to LDS.
template <int DT, int W> struct Tile {
  static constexpr int kVec = 16 / kBytes<DT>, kPerRow = W / kVec, kRows = 256 / kPerRow;
  static constexpr int kPasses = Traits<DT>::kChunk / kRows;
  static constexpr int kPitch = W + 16;   // elements
  Raw<4> r[kPasses];

  // row i is token t0 + dt * i, which exists within [lo, hi)
  __device__ __forceinline__ void load(const char* base, long row_stride, int D, int t0, int dt, int lo, int hi) {
    const int col = (threadIdx.x % kPerRow) * kVec, row = threadIdx.x / kPerRow;
    if (D % kVec == 0) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int t = t0 + dt * (row + i * kRows);
        r[i] = Raw<4>{0, 0, 0, 0};
        if (t >= lo && t < hi && col < D) r[i] = scan::load_wide<DT, kVec>(base + ((long)t * row_stride + col) * kBytes<DT>);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int t = t0 + dt * (row + i * kRows);
        const int avail = t >= lo && t < hi ? D - col : 0;
        r[i] = scan::load_vec<DT, kVec>(base + ((long)t * row_stride + col) * kBytes<DT>, avail);
      }
    }
  }
  __device__ __forceinline__ void store(typename Traits<DT>::Elem* lds) const {
    const int col = (threadIdx.x % kPerRow) * kVec, row = threadIdx.x / kPerRow;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) *reinterpret_cast<Raw<4>*>(lds + (row + i * kRows) * kPitch + col) = r[i];
  }
};

// 8 (4) consecutive elements of a row: an operand reduced along rows.
template <int DT>
__device__ __forceinline__ typename Traits<DT>::Frag row_frag(const typename Traits<DT>::Elem* p) {
  return *reinterpret_cast<const typename Traits<DT>::Frag*>(p);
}

// An operand reduced along tokens, lane m of a group of 16 having column m of
// 16: tokens 4 g .. (and 16 + 4 g ..) of a group of tokens.  Columns run in four
// pieces of 4, `step` elements apart.
template <int PITCH>
__device__ __forceinline__ bf16x8_t col_frag(const uint16_t* p, int lane, int step) {
  const int g = lane >> 4, m = lane & 15;
  const uint16_t* a = p + (4 * g + (m >> 2)) * PITCH + step * (m & 3);
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BC_LDS s16x4_t*)(uintptr_t)(uint32_t)(uintptr_t)(BC_LDS uint16_t*)a);
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BC_LDS s16x4_t*)(uintptr_t)(uint32_t)(uintptr_t)(BC_LDS uint16_t*)(a + 16 * PITCH));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int PITCH>
__device__ __forceinline__ f32x4_t col_frag(const float* p, int lane, int step) {
  const int g = lane >> 4, m = lane & 15;
  const float* a = p + 4 * g * PITCH + step * (m >> 2) + (m & 3);
  return f32x4_t{a[0], a[PITCH], a[2 * PITCH], a[3 * PITCH]};
}

// Token of element e of such an operand, within its group.
template <int DT>
__device__ __forceinline__ constexpr int col_token(int g, int e) { return (e >> 2) * 16 + 4 * g + (e & 3); }

// What a chunk's decays make, in LDS.
template <int CH> struct Decays {
  float hi[CH], lo[CH];   // L, log2
  float here[CH];         // exp(L_i)
  float rest[CH];         // exp(L_end - L_i), with the factor of k v^T
  float whole;            // exp(L_end)
};

// By one wave: the decay of row `lane`'s token (0 for rows past the chunk).
template <int CH>
__device__ __forceinline__ void make_decays(Decays<CH>* d, double l2, float kv, int lane, double& total) {
#pragma unroll
  for (int s = 1; s < CH; s *= 2) {
    const double o = __shfl_up(l2, s);
    if (lane >= s) l2 += o;
  }
  const double end = __shfl(l2, CH - 1);
  total += end;
  if (lane < CH) {
    const float hi = (float)l2;
    d->hi[lane] = hi;
    d->lo[lane] = (float)(l2 - (double)hi);
    d->here[lane] = exp2_parts(l2);
    d->rest[lane] = kv * exp2_parts(end - l2);
    if (lane == 0) d->whole = exp2_parts(end);
  }
}

template <int DT, int KP, int VP>
struct Smem {
  static constexpr int CH = Traits<DT>::kChunk, IT = CH / 16, kTiles = IT * (IT + 1) / 2;
  using E = typename Traits<DT>::Elem;
  alignas(16) E q[CH * Tile<DT, KP>::kPitch];
  alignas(16) E k[CH * Tile<DT, KP>::kPitch];
  alignas(16) E v[CH * Tile<DT, VP>::kPitch];
  alignas(16) char p[kTiles * 1024];   // score tiles: fp32, or two bf16 parts
  alignas(16) Decays<CH> dec[2];
  alignas(16) float dots[4][CH];
};

template <int DT, int KP, int VP, bool OUT>
__global__ __launch_bounds__(256, 2) void k_walk(Walk w) {
  using Tr = Traits<DT>;
  using Frag = typename Tr::Frag;
  using E = typename Tr::Elem;
  constexpr int CH = Tr::kChunk, KG = Tr::kGroup, IT = CH / 16, PG = CH / KG, TPG = KG / 16;
  constexpr int NT = VP / 64, KT = KP / 16, FE = KG / 4;
  constexpr int KPITCH = Tile<DT, KP>::kPitch, VPITCH = Tile<DT, VP>::kPitch;
  extern __shared__ char smem_raw[];
  auto& sm = *reinterpret_cast<Smem<DT, KP, VP>*>(smem_raw);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, m = lane & 15;
  const int seg = blockIdx.x % w.segs, nh = blockIdx.x / w.segs, n = nh / w.H, h = nh % w.H;
  const int len = w.lengths ? min(max(w.lengths[n], 0), w.T) : w.T;
  const int b = seg * w.seg, e = min(b + w.seg, w.T);
  const int chunks = (e - b + CH - 1) / CH;
  const int dt = w.rev ? -1 : 1, hi = min(e, len);

  const char* qp = w.q + (n * w.qs.n + (h / w.qd) * w.qs.h) * kBytes<DT>;
  const char* kp = w.k + (n * w.ks.n + (h / w.kd) * w.ks.h) * kBytes<DT>;
  const char* vp = w.v + (n * w.vs.n + (h / w.vd) * w.vs.h) * kBytes<DT>;
  const long g0 = n * w.gs.n + h * w.gs.h;

  Tile<DT, KP> tq, tk;
  Tile<DT, VP> tv;
  double l2 = 0.0, total = 0.0;
  auto first = [&](int c) { return w.rev ? e - 1 - c * CH : b + c * CH; };
  auto load = [&](int c) {
    const int t0 = first(c);
    if constexpr (OUT) tq.load(qp, w.qs.t, w.K, t0, dt, b, hi);
    tk.load(kp, w.ks.t, w.K, t0, dt, b, hi);
    tv.load(vp, w.vs.t, w.V, t0, dt, b, hi);
    if (wave == 0) {
      const int t = t0 + dt * lane, gt = w.rev ? t + 1 : t;
      l2 = 0.0;
      if (lane < CH && t >= b && t < e && gt < len) l2 = log2_decay(load_elem(w.gate, g0 + gt * w.gs.t, w.gate_f32), w.form);
    }
  };

  // the wave's columns: lane m of tile nt has column c0 + vcol(nt, m), so that a
  // lane's outputs of both tiles are consecutive
  const int c0 = wave * 16 * NT;
  auto vcol = [&](int nt, int mm) { return NT == 2 ? 8 * (mm >> 2) + 4 * nt + (mm & 3) : mm; };
  constexpr int VSTEP = NT == 2 ? 8 : 4;
  // rows of S that lane group g holds of tile kt: krow(kt) + 0..3
  auto krow = [&](int kt, int gg) { return DT == kBF16 ? 32 * (kt >> 1) + 8 * gg + 4 * (kt & 1) : 16 * kt + 4 * gg; };
  constexpr int KSTEP = DT == kBF16 ? 8 : 4;
  auto kcol = [&](int kt) { return DT == kBF16 ? 32 * (kt >> 1) + 4 * (kt & 1) : 16 * kt; };

  f32x4_t S[KT][NT];
  {
    const float* p = w.init ? w.init + nh * w.init_nh + seg * w.init_seg : nullptr;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int kk = krow(kt, g) + r, vv = c0 + vcol(nt, m);
          S[kt][nt][r] = p && kk < w.K && vv < w.V ? p[kk * w.sk + vv * w.sv] : 0.0f;
        }
  }
  auto put_state = [&](float* p, float f) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int kk = krow(kt, g) + r, vv = c0 + vcol(nt, m);
          if (kk < w.K && vv < w.V) p[kk * w.sk + vv * w.sv] = S[kt][nt][r] * f;
        }
  };

  load(0);
  if (wave == 0) make_decays<CH>(&sm.dec[0], l2, w.kv, lane, total);
  for (int c = 0; c < chunks; ++c) {
    const int t0 = first(c);
    // nothing of the chunk exists: its outputs are zero, the state stays
    const bool dead = (w.rev ? t0 - CH + 1 : t0) >= len;
    const Decays<CH>& d = sm.dec[c & 1];
    if (!dead) {
      if constexpr (OUT) tq.store(sm.q);
      tk.store(sm.k);
      tv.store(sm.v);
    }
    __syncthreads();
    if (c + 1 < chunks) load(c + 1);
    if constexpr (OUT) {
      if (w.save && (t0 - b) % w.span == 0 && t0 % w.span == 0) put_state(w.save + nh * w.save_nh + (t0 / w.span) * (long)w.K * w.V, 1.0f);
    }
    f32x4_t acc[IT][NT];
    Frag vf[PG][NT];
    if (!dead) {
      if constexpr (OUT) {
        // scores of the causal tiles, transposed: rows j, columns i
        for (int i = wave; i < IT * (IT + 1) / 2; i += 4) {
          const int it = (i >= 1) + (i >= 3) + (i >= 6), jt = i - it * (it + 1) / 2;
          f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kg = 0; kg < KP / KG; ++kg)
            s = mma(row_frag<DT>(sm.k + (jt * 16 + m) * KPITCH + kg * KG + g * FE),
                    row_frag<DT>(sm.q + (it * 16 + m) * KPITCH + kg * KG + g * FE), s);
          const int ii = it * 16 + m, jj = jt * 16 + 4 * g;
          const float ih = d.hi[ii], il = d.lo[ii];
          const f32x4_t jh = *reinterpret_cast<const f32x4_t*>(&d.hi[jj]), jl = *reinterpret_cast<const f32x4_t*>(&d.lo[jj]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[r] = jj + r <= ii ? s[r] * (w.kv * __builtin_amdgcn_exp2f((ih - jh[r]) + (il - jl[r]))) : 0.0f;
          if constexpr (DT == kBF16) {
            bf16x4_t h4, l4;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              h4[r] = (__bf16)s[r];
              l4[r] = (__bf16)(s[r] - (float)h4[r]);
            }
            reinterpret_cast<bf16x4_t*>(sm.p)[i * 128 + lane] = h4;
            reinterpret_cast<bf16x4_t*>(sm.p)[i * 128 + 64 + lane] = l4;
          } else {
            reinterpret_cast<f32x4_t*>(sm.p)[i * 64 + lane] = s;
          }
        }
        // what the state before the chunk adds: rows v, columns i
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[it][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kg = 0; kg < KP / KG; ++kg) {
          Split<DT, 2> sp[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x[FE];
#pragma unroll
            for (int q = 0; q < FE; ++q) x[q] = S[kg * TPG + q / 4][nt][q & 3];
            sp[nt] = split<2>(x);
          }
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const Frag f = row_frag<DT>(sm.q + (it * 16 + m) * KPITCH + kg * KG + g * FE);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[it][nt] = mma<DT, 2>(sp[nt], f, acc[it][nt]);
          }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const float f = d.here[it * 16 + m];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[it][nt] *= f;
        }
      }
#pragma unroll
      for (int p = 0; p < PG; ++p)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          vf[p][nt] = col_frag<VPITCH>(sm.v + p * KG * VPITCH + c0 + (NT == 2 ? 4 * nt : 0), lane, VSTEP);
    }
    if constexpr (OUT) {
      __syncthreads();
      if (!dead) {
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int p = 0; p < PG; ++p) {
            if (p * TPG > it) continue;
            Split<DT, 2> pf;
            if constexpr (DT == kBF16) {
              const bf16x4_t z = {};
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int i = it * (it + 1) / 2 + 2 * p;
                const bf16x4_t a = reinterpret_cast<const bf16x4_t*>(sm.p)[i * 128 + u * 64 + lane];
                const bf16x4_t bb = 2 * p + 1 <= it ? reinterpret_cast<const bf16x4_t*>(sm.p)[(i + 1) * 128 + u * 64 + lane] : z;
                pf.part[u] = __builtin_shufflevector(a, bb, 0, 1, 2, 3, 4, 5, 6, 7);
              }
            } else {
              pf.part[0] = reinterpret_cast<const f32x4_t*>(sm.p)[(it * (it + 1) / 2 + p) * 64 + lane];
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[it][nt] = mma<DT, 2>(vf[p][nt], pf, acc[it][nt]);
          }
      }
      // outputs: a lane has 4 NT consecutive columns of row it * 16 + m
      constexpr int V = 4 * NT;
      const int col = c0 + (NT == 2 ? 8 * g : 4 * g), avail = w.V - col;
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int t = t0 + dt * (it * 16 + m);
        const bool exists = t >= b && t < e, live = exists && t < len;
        float o[V], dot = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q) o[q] = live ? acc[it][q / 4][q & 3] * w.scale : 0.0f;
        if (w.x && live) {
          const Raw<scan::kWords<DT, V>> xr =
              scan::load_vec<DT, V>(w.x + (n * w.xs.n + t * w.xs.t + (h / w.xd) * w.xs.h + col) * kBytes<DT>, avail);
#pragma unroll
          for (int q = 0; q < V; ++q) dot = fmaf(o[q], scan::elem<DT, V>(xr, q), dot);
        }
        if (exists && avail > 0) {
          const long at = n * w.ys.n + t * w.ys.t + h * w.ys.h + col;
          if (DT == kF32 || w.y_f32) scan::store_vec<kF32, V>(w.y + at * 4, avail, o);
          else scan::store_vec<kBF16, V>(w.y + at * 2, avail, o);
        }
        if (w.x) {
          dot += __shfl_xor(dot, 16);
          dot += __shfl_xor(dot, 32);
          if (g == 0) sm.dots[wave][it * 16 + m] = dot;
        }
      }
    }
    if (!dead) {
      const float whole = d.whole;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) S[kt][nt] *= whole;
#pragma unroll
      for (int p = 0; p < PG; ++p) {
        Split<DT, 3> sp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[FE];
#pragma unroll
          for (int q = 0; q < FE; ++q) x[q] = (float)vf[p][nt][q] * d.rest[p * KG + col_token<DT>(g, q)];
          sp[nt] = split<3>(x);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const Frag f = col_frag<KPITCH>(sm.k + p * KG * KPITCH + kcol(kt), lane, KSTEP);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) S[kt][nt] = mma<DT, 3>(f, sp[nt], S[kt][nt]);
        }
      }
    }
    if (c + 1 < chunks && wave == 0) make_decays<CH>(&sm.dec[(c + 1) & 1], l2, w.kv, lane, total);
    __syncthreads();
    if constexpr (OUT) {
      if (w.x && tid < CH) {
        const int t = t0 + dt * tid;
        if (t >= b && t < e) w.dots[(long)nh * w.T + t] = (sm.dots[0][tid] + sm.dots[1][tid]) + (sm.dots[2][tid] + sm.dots[3][tid]);
      }
    }
  }
  if (w.last) {
    float f = 1.0f;
    if (w.last_a0 && len > 0) f = exp2_parts(log2_decay(load_elem(w.gate, g0, w.gate_f32), w.form));
    put_state(w.last + nh * w.last_nh + min(seg * w.last_seg, w.last_max), f);
  }
  if (w.last2) put_state(w.last2 + nh * w.last2_nh, 1.0f);
  if (w.decay && tid == 0) w.decay[(long)nh * w.segs + seg] = exp2_parts(total);
}

template <int DT, int KP, int VP>
hipError_t launch_walk_sized(const Walk& w, hipStream_t s) {
  auto go = [&](auto kernel, size_t lds) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((long)w.N * w.H * w.segs)), dim3(256), (unsigned)lds, s, w);
    return hipGetLastError();
  };
  return w.y ? go(k_walk<DT, KP, VP, true>, sizeof(Smem<DT, KP, VP>)) : go(k_walk<DT, KP, VP, false>, sizeof(Smem<DT, KP, VP>));
}

template <int DT>
hipError_t launch_walk_dt(const Walk& w, hipStream_t s) {
  if (w.K <= 64) return w.V <= 64 ? launch_walk_sized<DT, 64, 64>(w, s) : launch_walk_sized<DT, 64, 128>(w, s);
  return w.V <= 64 ? launch_walk_sized<DT, 128, 64>(w, s) : launch_walk_sized<DT, 128, 128>(w, s);
}

}  // namespace
}  // namespace linattn
}  // namespace bc
