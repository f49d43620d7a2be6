// The walk of linear attention over a segment (bc_linattn.hpp), on MFMA.
//
// A block of four waves takes a segment of one sequence and head, chunk by chunk of
// 32 tokens: q, k and v of a chunk go through LDS, each wave owns 16 or 32 of the
// state's columns (v's), which stay in its registers as fp32 accumulators, and the
// chunk's scores, one 16 x 16 tile at a time, are shared through LDS.
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
// scores and S into two (to 2^-16 of themselves; they make outputs of 2^-8, and products
// with q and k whose sums, the gates' gradients, are 5e-6 to 2e-5 off as a whole also
// where a gate is fp32: less than the inputs' own roundings move them), the
// decayed v that the state takes in into three (2^-24: the state is fp32).
// fp32: the fp32 matrix instruction.
//
// What bounds it: the walk itself, a chunk's steps one after the other with two waves
// a SIMD (S takes 64 registers of a wave, the chunk on its way 24).  bf16, rows of
// 128, 64 heads of 4096 tokens in 512 segments: 79 us for outputs (300 MB, 3.8 TB/s;
// the matrix units are busy 40 % of the time, the vector units 44 %), 44 us for states
// alone (167 MB, 3.8 TB/s); 8 heads of 65536 tokens, 172 and 86 us.  fp32, 8 heads of
// 8192 tokens in 256 segments, rows of 64 and 128: 40 and 21 us (the matrix units 49 %
// busy, 61 to 65 % where two walks share a launch).  Rows that are not whole vectors (VEC false)
// cost about a sixth more: in training 64 heads of 4096 with 128 x 122 in place of
// 128 x 120, 488 us for 420.  Chunks of 64 tokens halve the work on
// S but leave no registers: 487 us for a training call of the first size, of 32 436.
// Two places in LDS for a chunk's rows, and so a barrier less, make no difference.
// No vector register is spilled; of the scalar ones (buffers, strides, bounds) 5 to 265
// live in lanes of a vector register, and some 40 to 55 of a chunk's 560 to 800
// instructions fetch and keep them.
#pragma once
#include <initializer_list>

#include "bc_common.hpp"
#include "bc_linattn.hpp"

namespace bc {
namespace linattn {
namespace {

template <int DT> struct Traits;
template <> struct Traits<kBF16> {
  static constexpr int kGroup = 32;   // the reduction of one operand pair
  using Frag = bf16x8_t;
  using Elem = uint16_t;
};
template <> struct Traits<kF32> {
  static constexpr int kGroup = 16;
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

// Two values to a bf16 pair, nearest even, in one instruction.
__device__ __forceinline__ uint32_t round_pair(float lo, float hi) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

// fp32 values as a sum of P operands.
template <int DT, int P> struct Split {
  typename Traits<DT>::Frag part[DT == kBF16 ? P : 1];
};
// x: the values of an operand as two tiles of accumulators.  What a part leaves is the
// tile less that part, exactly: the matrix unit subtracts (minus_of).
template <int P>
__device__ __forceinline__ Split<kBF16, P> split(const f32x4_t (&x)[2], const bf16x8_t (&minus)[2]) {
  Split<kBF16, P> s;
  f32x4_t rest[2] = {x[0], x[1]};
#pragma unroll
  for (int p = 0; p < P; ++p) {
    Raw<4> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = round_pair(rest[i / 2][2 * (i & 1)], rest[i / 2][2 * (i & 1) + 1]);
    s.part[p] = __builtin_bit_cast(bf16x8_t, w);
    if (p + 1 < P) {
      rest[0] = mma(minus[0], s.part[p], rest[0]);
      rest[1] = mma(minus[1], s.part[p], rest[1]);
    }
  }
  return s;
}
template <int P>
__device__ __forceinline__ Split<kF32, P> split(const f32x4_t (&x)[1], const f32x4_t (&)[2]) {
  Split<kF32, P> s;
  s.part[0] = x[0];
  return s;
}
// The operands that take an operand from its two tiles: row 4 g + r of tile i is the
// operand's element 8 g + 4 i + r, so there they have -1, and zeros elsewhere.
template <int DT> __device__ __forceinline__ void minus_of(typename Traits<DT>::Frag (&minus)[2], int lane) {
  if constexpr (DT == kBF16) {
    const bool on = lane >> 4 == (lane & 15) >> 2;
    const Raw<2> w = {on && (lane & 2) == 0 ? (lane & 1 ? 0xbf800000u : 0xbf80u) : 0u,
                      on && (lane & 2) != 0 ? (lane & 1 ? 0xbf800000u : 0xbf80u) : 0u};
    minus[0] = __builtin_bit_cast(bf16x8_t, Raw<4>{w[0], w[1], 0u, 0u});
    minus[1] = __builtin_bit_cast(bf16x8_t, Raw<4>{0u, 0u, w[0], w[1]});
  }
}
// (fp32 needs but one; smaller parts are added first)
template <int DT, int P> constexpr int kParts = DT == kBF16 ? P : 1;

// Rows [0, rows) of `width` bytes, `step` >= width apart, from p: what a buffer
// operation reads past them is zero, and what it would write there is dropped.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const char* p, int rows, int step, int width) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, rows > 0 ? (rows - 1) * step + width : 0, 0x00020000);
}
constexpr uint32_t kNoColumn = 0x80000000u;   // past every row: such offsets stay below 2^32

// W words at `at`; of 8 the last four only where the row has them (both).
template <int W> __device__ __forceinline__ Raw<W> buffer_load(__amdgpu_buffer_rsrc_t rs, uint32_t at, bool both = true) {
  if constexpr (W == 2) return __builtin_bit_cast(Raw<2>, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)at, 0, 0));
  else if constexpr (W == 4) return __builtin_bit_cast(Raw<4>, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at, 0, 0));
  else {
    const Raw<4> a = buffer_load<4>(rs, at), b = buffer_load<4>(rs, both ? at + 16 : kNoColumn);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
template <int W> __device__ __forceinline__ void buffer_store(__amdgpu_buffer_rsrc_t rs, uint32_t at, const Raw<W>& v, bool both = true) {
  if constexpr (W == 2) __builtin_amdgcn_raw_buffer_store_b64(v, rs, (int)at, 0, 0);
  else if constexpr (W == 4) __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)at, 0, 0);
  else {
    buffer_store<4>(rs, at, __builtin_shufflevector(v, v, 0, 1, 2, 3));
    buffer_store<4>(rs, both ? at + 16 : kNoColumn, __builtin_shufflevector(v, v, 4, 5, 6, 7));
  }
}

// Element e of the result is element e + over of v, zero past its end; over <= V.
template <int DT, int V>
__device__ __forceinline__ Raw<scan::kWords<DT, V>> shift_down(Raw<scan::kWords<DT, V>> v, int over) {
  constexpr int W = scan::kWords<DT, V>;
  if constexpr (DT == kBF16) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = over & 1 ? __builtin_amdgcn_alignbit(i + 1 < W ? v[i + 1] : 0u, v[i], 16) : v[i];
    over >>= 1;
  }
#pragma unroll
  for (int s = 1; s <= W; s *= 2)
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = over & s ? (i + s < W ? v[i + s] : 0u) : v[i];
  return v;
}

// A chunk's rows of one operand: from memory to registers, then to LDS.
template <int DT, int W, int THREADS> struct Tile {
  static constexpr int kVec = 16 / kBytes<DT>, kPerRow = W / kVec, kRows = THREADS / kPerRow;
  static constexpr int CH = kChunk, kPasses = (CH + kRows - 1) / kRows;
  static constexpr int kPitch = W + 16;   // elements
  static_assert(kPasses * kRows == CH || kRows > CH, "whole passes, or one of which threads are idle");
  Raw<4> r[kPasses];

  static __device__ __forceinline__ int col() { return (threadIdx.x % kPerRow) * kVec; }
  static __device__ __forceinline__ bool busy() { return kRows <= CH || threadIdx.x < CH * kPerRow; }
  // row i of the tile is token t0 + i, or t0 + CH - 1 - i (rev)
  static __device__ __forceinline__ int row(int pass, bool rev) {
    const int k = threadIdx.x / kPerRow + pass * kRows;
    return rev ? CH - 1 - k : k;
  }

  // the rows of the tile's first token on, `from` bytes behind rs
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, int step, int from, int D, bool rev) {
    const uint32_t at = (col() < D && busy() ? (uint32_t)(row(0, rev) * step + col() * kBytes<DT>) : kNoColumn) + (uint32_t)from;
    const int skip = rev ? -kRows * step : kRows * step;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) r[i] = buffer_load<4>(rs, at + (uint32_t)(i * skip));
  }
  // Any rows, tokens from hi (> t0) on do not exist.  A vector past the row's end is the
  // row's last one, and that of a token that does not exist the last token's: every
  // load is whole and in range, none waits for another, and settle() puts in order
  // what has arrived.  (Rows shorter than a vector: element by element.)
  __device__ __forceinline__ void load(const char* base, long row_stride, int D, int t0, bool rev, int hi) {
    const int c = min(col(), D - kVec);
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int t = t0 + row(i, rev);
      if (D < kVec) r[i] = scan::load_vec<DT, kVec>(base + ((long)t * row_stride + col()) * kBytes<DT>, t < hi && busy() ? D - col() : 0);
      else r[i] = scan::load_wide<DT, kVec>(base + ((long)max(min(t, hi - 1), t0) * row_stride + c) * kBytes<DT>);
    }
  }
  __device__ __forceinline__ void settle(int D, int t0, bool rev, int hi) {
    if (D < kVec) return;
    const int over = min(col() - min(col(), D - kVec), kVec);
#pragma unroll
    for (int i = 0; i < kPasses; ++i) r[i] = shift_down<DT, kVec>(r[i], t0 + row(i, rev) < hi ? over : kVec);
  }
  __device__ __forceinline__ void store(typename Traits<DT>::Elem* lds) const {
    if (!busy()) return;
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
      *reinterpret_cast<Raw<4>*>(lds + (threadIdx.x / kPerRow + i * kRows) * kPitch + col()) = r[i];
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

constexpr int kAhead = 32;   // chunks whose decays are made at a time

template <int DT, int KP, int VP, int NT>
struct Smem {
  static constexpr int CH = kChunk, IT = CH / 16, kTiles = IT * (IT + 1) / 2, kWaves = VP / 16 / NT;
  using E = typename Traits<DT>::Elem;
  alignas(16) E q[CH * (KP + 16)];
  alignas(16) E k[CH * (KP + 16)];
  alignas(16) E v[CH * (VP + 16)];
  alignas(16) char p[kTiles * 1024];   // score tiles: fp32, or two bf16 parts
  // What the decays make, of kAhead chunks: rows {hi, lo, here, rest}, with L the
  // running sum of log2 a over the chunk up to a token, in the order of the walk:
  // hi + lo = L, here = 2^L, rest = 2^(end - L) times the factor of k v^T; and 2^end.
  alignas(16) float dec[kAhead][4][CH];
  float whole[kAhead];
  double totals[kWaves];
  alignas(16) float dots[kWaves][CH];
};

// MODE: the states alone, with outputs, or with outputs and their products with x.
constexpr int kStates = 0, kOut = 1, kOutDots = 2;

template <int DT, int KP, int VP, int NT, int MODE, bool VEC>
__device__ __forceinline__ void walk(const Walk& w, int block, char* smem_raw) {
  constexpr bool OUT = MODE != kStates, DOTS = MODE == kOutDots;
  using Tr = Traits<DT>;
  using Frag = typename Tr::Frag;
  using SM = Smem<DT, KP, VP, NT>;
  constexpr int CH = kChunk, KG = Tr::kGroup, IT = CH / 16, PG = CH / KG, TPG = KG / 16;
  constexpr int KT = KP / 16, FE = KG / 4, THREADS = VP / NT * 4, WAVES = VP / 16 / NT;
  constexpr int KPITCH = KP + 16, VPITCH = VP + 16;
  SM& sm = *reinterpret_cast<SM*>(smem_raw);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, m = lane & 15;
  const int seg = block % w.segs, nh = block / w.segs, n = nh / w.H, h = nh % w.H;
  const int len = w.lengths ? min(max(w.lengths[n], 0), w.T) : w.T;
  const int b = seg * w.seg, e = min(b + w.seg, w.T);
  const int chunks = (e - b + CH - 1) / CH;
  const bool rev = w.rev;
  const int hi = min(e, len);

  const char* qp = w.q + (n * w.qs.n + (h / w.qd) * w.qs.h) * kBytes<DT>;
  const char* kp = w.k + (n * w.ks.n + (h / w.kd) * w.ks.h) * kBytes<DT>;
  const char* vp = w.v + (n * w.vs.n + (h / w.vd) * w.vs.h) * kBytes<DT>;

  Tile<DT, KP, THREADS> tq, tk;
  Tile<DT, VP, THREADS> tv;
  // the first token of chunk c in memory (its last in time, rev)
  auto first = [&](int c) { return b + (rev ? chunks - 1 - c : c) * CH; };
  // a chunk of which nothing exists: its outputs are zero, the state stays
  auto dead = [&](int t0) { return t0 >= len; };
  // VEC: buffers of the rows of kAhead chunks, from the first one in memory on; a
  // chunk's rows are an offset into them
  const int sq = (int)w.qs.t * kBytes<DT>, skk = (int)w.ks.t * kBytes<DT>, svv = (int)w.vs.t * kBytes<DT>;
  __amdgpu_buffer_rsrc_t rq, rk, rv;
  int low = 0;
  auto lowest = [&](int c) { return rev ? first(min(c + kAhead, chunks) - 1) : first(c); };
  auto load = [&](int c) {
    if (c >= chunks) return;
    if (VEC && c % kAhead == 0) {
      low = lowest(c);
      const int rows = min(hi - low, kAhead * CH);
      if constexpr (OUT) rq = rows_of(qp + low * w.qs.t * kBytes<DT>, rows, sq, w.K * kBytes<DT>);
      rk = rows_of(kp + low * w.ks.t * kBytes<DT>, rows, skk, w.K * kBytes<DT>);
      rv = rows_of(vp + low * w.vs.t * kBytes<DT>, rows, svv, w.V * kBytes<DT>);
    }
    const int t0 = first(c);
    if (dead(t0)) return;
    if constexpr (VEC) {
      if constexpr (OUT) tq.load(rq, sq, (t0 - low) * sq, w.K, rev);
      tk.load(rk, skk, (t0 - low) * skk, w.K, rev);
      tv.load(rv, svv, (t0 - low) * svv, w.V, rev);
    } else {
      if constexpr (OUT) tq.load(qp, w.qs.t, w.K, t0, rev, hi);
      tk.load(kp, w.ks.t, w.K, t0, rev, hi);
      tv.load(vp, w.vs.t, w.V, t0, rev, hi);
    }
  };

  // The decays of chunks c .. c + kAhead - 1, half a wave each.  Backward in time a
  // token's own decay lies behind it: the next one's is between.
  double total = 0.0;
  auto decays = [&](int c) {
    const int half = lane >> 5, i = lane & 31;
    constexpr int N2 = kAhead / 2 / WAVES;
    float gate[N2];
    bool on[N2];
#pragma unroll
    for (int u = 0; u < N2; ++u) {
      const int ch = c + 2 * (wave + u * WAVES) + half, t = first(ch) + (rev ? CH - i : i);
      on[u] = ch < chunks && t < len;
      gate[u] = 0.0f;
      if (on[u]) gate[u] = load_elem(w.gate, n * w.gs.n + t * w.gs.t + h * w.gs.h, w.gate_f32);
    }
#pragma unroll 1
    for (int u = 0; u < N2; ++u) {
      const int at = 2 * (wave + u * WAVES) + half;
      if (c + 2 * (wave + u * WAVES) >= chunks) break;
      float gu = gate[0];
      bool ou = on[0];
#pragma unroll
      for (int v = 1; v < N2; ++v) {
        gu = u == v ? gate[v] : gu;
        ou = u == v ? on[v] : ou;
      }
      double l2 = ou ? log2_decay(gu, w.form) : 0.0;
#pragma unroll
      for (int s = 1; s < CH; s *= 2) {
        const double o = __shfl_up(l2, s, 32);
        if (i >= s) l2 += o;
      }
      const double end = __shfl(l2, 31, 32);
      total += end;
      const float hi = (float)l2;
      float(&d)[4][CH] = sm.dec[at];
      d[0][i] = hi;
      d[1][i] = (float)(l2 - (double)hi);
      d[2][i] = exp2_parts(l2);
      d[3][i] = w.kv * exp2_parts(end - l2);
      if (i == 0) sm.whole[at] = exp2_parts(end);
    }
  };

  // the wave's 16 columns of the state, c0 + m; its rows that lane group g holds
  // of tile kt: krow(kt, g) + 0..3, so that an operand's are consecutive
  const int c0 = wave * 16 * NT;
  auto vcol = [&](int nt, int mm) { return NT == 2 ? 8 * (mm >> 2) + 4 * nt + (mm & 3) : mm; };
  constexpr int VSTEP = 4 * NT;
  auto krow = [&](int kt, int gg) { return DT == kBF16 ? 32 * (kt >> 1) + 8 * gg + 4 * (kt & 1) : 16 * kt + 4 * gg; };
  constexpr int KSTEP = DT == kBF16 ? 8 : 4;
  auto kcol = [&](int kt) { return DT == kBF16 ? 32 * (kt >> 1) + 4 * (kt & 1) : 16 * kt; };

  load(0);
  // A state in memory: element (kk, vv) at kk sk + vv sv.  What the tile has past K
  // rows or V columns reads as zero and is not written.
  const int sk = w.rows_first ? w.V : 1, sv = w.rows_first ? 1 : w.K, cells = w.K * w.V * 4;
  auto cell = [&](int kk, int vv) { return kk < w.K && vv < w.V ? (uint32_t)(kk * sk + vv * sv) * 4u : kNoColumn; };
  f32x4_t S[KT][NT];
  if (w.init) {
    const auto rs = rows_of(reinterpret_cast<const char*>(w.init + nh * w.init_nh + seg * w.init_seg), 1, 0, cells);
    if (VEC && sk == 1) {   // four rows are one vector
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          S[kt][nt] = __builtin_bit_cast(f32x4_t, buffer_load<4>(rs, cell(krow(kt, g), c0 + vcol(nt, m))));
    } else {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            S[kt][nt][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (int)cell(krow(kt, g) + r, c0 + vcol(nt, m)), 0, 0));
    }
  } else {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) S[kt][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  decays(0);
  auto put_state = [&](float* p, float f) {
    const auto rs = rows_of(reinterpret_cast<const char*>(p), 1, 0, cells);
    // (offsets made here, not kept from above through the loop: 64 registers)
    int gg = g, mm = m;
    asm volatile("" : "+v"(gg), "+v"(mm));
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[kt][nt][r] * f), rs,
                                                (int)cell(krow(kt, gg) + r, c0 + vcol(nt, mm)), 0, 0);
  };

  if (w.first) put_state(w.first + nh * w.last2_nh, 1.0f);

  Frag minus[2];
  minus_of<DT>(minus, lane);
  const float reach = w.kv * w.scale;   // of the scores
  const int out_bytes = DT == kF32 || w.y_f32 ? 4 : 2;
  char* yp = OUT ? w.y + (n * w.ys.n + h * w.ys.h) * out_bytes : nullptr;
  const char* xp = DOTS ? w.x + (n * w.xs.n + (h / w.xd) * w.xs.h) * kBytes<DT> : nullptr;
  const int ystep = (int)w.ys.t * out_bytes, xstep = (int)w.xs.t * kBytes<DT>;
  __amdgpu_buffer_rsrc_t ry, rx;
  int out_low = 0;
  for (int c = 0; c < chunks; ++c) {
    const int t0 = first(c);
    const bool live = !dead(t0);
    if (c % kAhead == 0) {
      if (c > 0) decays(c);
      if constexpr (OUT && VEC) {
        out_low = lowest(c);
        ry = rows_of(yp + out_low * w.ys.t * out_bytes, min(e - out_low, kAhead * CH), ystep, w.V * out_bytes);
        if constexpr (DOTS) rx = rows_of(xp + out_low * w.xs.t * kBytes<DT>, min(hi - out_low, kAhead * CH), xstep, w.V * kBytes<DT>);
      }
    }
    const float(&d)[4][CH] = sm.dec[c % kAhead];
    if (live) {
      if constexpr (!VEC) {
        if constexpr (OUT) tq.settle(w.K, t0, rev, hi);
        tk.settle(w.K, t0, rev, hi);
        tv.settle(w.V, t0, rev, hi);
      }
      if constexpr (OUT) tq.store(sm.q);
      tk.store(sm.k);
      tv.store(sm.v);
    }
    __syncthreads();
    const float whole = sm.whole[c % kAhead];
    load(c + 1);
    __builtin_amdgcn_sched_barrier(0);
    // the rows that outputs are multiplied with, on their way from here
    constexpr int V = 4 * NT;
    const int col = c0 + V * g, avail = w.V - col;
    const bool both = DT != kF32 || avail > 4;   // (whole vectors of fp32 are half a lane's columns)
    Raw<scan::kWords<DT, V>> x[DOTS ? IT : 1];
    if constexpr (DOTS) {
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int row = rev ? CH - 1 - it * 16 - m : it * 16 + m;
        if constexpr (VEC) x[it] = buffer_load<scan::kWords<DT, V>>(rx, avail > 0 ? (uint32_t)((t0 - out_low + row) * xstep + col * kBytes<DT>) : kNoColumn, both);
        else if (w.V < V) x[it] = scan::load_vec<DT, V>(xp + ((t0 + row) * w.xs.t + col) * kBytes<DT>, t0 + row < hi ? avail : 0);
        else x[it] = scan::load_wide<DT, V>(xp + (max(min(t0 + row, hi - 1), t0) * w.xs.t + min(col, w.V - V)) * kBytes<DT>);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    f32x4_t acc[IT][NT];
    Frag vf[PG][NT];
    if (live) {
      if constexpr (OUT) {
        // scores of the causal tiles, transposed: rows j, columns i
        for (int i = wave; i < SM::kTiles; i += WAVES) {
          const int it = (i >= 1) + (i >= 3) + (i >= 6), jt = i - it * (it + 1) / 2;
          f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kg = 0; kg < KP / KG; ++kg)
            s = mma(row_frag<DT>(sm.k + (jt * 16 + m) * KPITCH + kg * KG + g * FE),
                    row_frag<DT>(sm.q + (it * 16 + m) * KPITCH + kg * KG + g * FE), s);
          const int ii = it * 16 + m, jj = jt * 16 + 4 * g;
          const float ih = d[0][ii], il = d[1][ii];
          const f32x4_t jh = *reinterpret_cast<const f32x4_t*>(&d[0][jj]), jl = *reinterpret_cast<const f32x4_t*>(&d[1][jj]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[r] = jj + r <= ii ? s[r] * (reach * __builtin_amdgcn_exp2f((ih - jh[r]) + (il - jl[r]))) : 0.0f;
          if constexpr (DT == kBF16) {
            Raw<2> h2, l2;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              h2[r] = round_pair(s[2 * r], s[2 * r + 1]);
              l2[r] = round_pair(s[2 * r] - __uint_as_float(h2[r] << 16), s[2 * r + 1] - __uint_as_float(h2[r] & 0xffff0000u));
            }
            reinterpret_cast<Raw<2>*>(sm.p)[i * 128 + lane] = h2;
            reinterpret_cast<Raw<2>*>(sm.p)[i * 128 + 64 + lane] = l2;
          } else {
            reinterpret_cast<f32x4_t*>(sm.p)[i * 64 + lane] = s;
          }
        }
        // what the state before the chunk adds: rows v, columns i.  (This stretch has the
        // most to issue: a wave in it goes before another block's, 2 % of a training call.)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[it][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kg = 0; kg < KP / KG; ++kg) {
          Split<DT, 2> sp[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f32x4_t x[TPG];
#pragma unroll
            for (int u = 0; u < TPG; ++u) x[u] = S[kg * TPG + u][nt];
            sp[nt] = split<2>(x, minus);
          }
          Frag f[IT];
#pragma unroll
          for (int it = 0; it < IT; ++it) f[it] = row_frag<DT>(sm.q + (it * 16 + m) * KPITCH + kg * KG + g * FE);
#pragma unroll
          for (int part = kParts<DT, 2> - 1; part >= 0; --part)
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) acc[it][nt] = mma(sp[nt].part[part], f[it], acc[it][nt]);
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const float f = w.scale * d[2][it * 16 + m];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[it][nt] *= f;
        }
      }
#pragma unroll
      for (int p = 0; p < PG; ++p)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) vf[p][nt] = col_frag<VPITCH>(sm.v + p * KG * VPITCH + c0 + 4 * nt * (NT - 1), lane, VSTEP);
    }
    if constexpr (OUT) {
      __builtin_amdgcn_s_setprio(0);
      __syncthreads();
      if (live) {
#pragma unroll
        for (int p = 0; p < PG; ++p) {
          Split<DT, 2> pf[IT];
#pragma unroll
          for (int it = p * TPG; it < IT; ++it) {
            if constexpr (DT == kBF16) {
              const bf16x4_t z = {};
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int i = it * (it + 1) / 2 + 2 * p;
                const bf16x4_t a = reinterpret_cast<const bf16x4_t*>(sm.p)[i * 128 + u * 64 + lane];
                const bf16x4_t bb = 2 * p + 1 <= it ? reinterpret_cast<const bf16x4_t*>(sm.p)[(i + 1) * 128 + u * 64 + lane] : z;
                pf[it].part[u] = __builtin_shufflevector(a, bb, 0, 1, 2, 3, 4, 5, 6, 7);
              }
            } else {
              pf[it].part[0] = reinterpret_cast<const f32x4_t*>(sm.p)[(it * (it + 1) / 2 + p) * 64 + lane];
            }
          }
#pragma unroll
          for (int part = kParts<DT, 2> - 1; part >= 0; --part)
#pragma unroll
            for (int it = p * TPG; it < IT; ++it)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) acc[it][nt] = mma(vf[p][nt], pf[it].part[part], acc[it][nt]);
        }
      }
      // outputs: a lane has V consecutive columns of row it * 16 + m
      if (t0 + CH > hi) {   // rows that do not exist
#pragma unroll
        for (int it = 0; it < IT; ++it)
          if (t0 + (rev ? CH - 1 - it * 16 - m : it * 16 + m) >= hi)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[it][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int row = rev ? CH - 1 - it * 16 - m : it * 16 + m;
        float o[V];
#pragma unroll
        for (int u = 0; u < V; ++u) o[u] = acc[it][u / 4][u & 3];
        if constexpr (VEC) {
          if (out_bytes == 4)
            buffer_store<V>(ry, avail > 0 ? (uint32_t)((t0 - out_low + row) * ystep + col * 4) : kNoColumn, scan::rounded<kF32, V>(o), both);
          else
            buffer_store<V / 2>(ry, avail > 0 ? (uint32_t)((t0 - out_low + row) * ystep + col * 2) : kNoColumn, scan::rounded<kBF16, V>(o));
        } else if (t0 + row < e && avail > 0) {
          const long at = ((t0 + row) * w.ys.t + col) * out_bytes;
          if (out_bytes == 4) scan::store_vec<kF32, V>(yp + at, avail, o);
          else scan::store_vec<kBF16, V>(yp + at, avail, o);
        }
        if constexpr (DOTS) {
          float dot = 0.0f;
          if (!VEC && w.V >= V) {   // (as Tile::settle)
            const int over = min(col - min(col, w.V - V), V);
            x[it] = shift_down<DT, V>(x[it], t0 + row < hi ? over : V);
          }
#pragma unroll
          for (int u = 0; u < V; ++u) dot = fmaf(o[u], scan::elem<DT, V>(x[it], u), dot);
          dot = pair32_sum(pair16_sum(dot));
          if (g == 0) sm.dots[wave][it * 16 + m] = dot;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (live) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) S[kt][nt] *= whole;
#pragma unroll
      for (int p = 0; p < PG; ++p) {
        Split<DT, 3> sp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4_t x[TPG];
#pragma unroll
          for (int u = 0; u < FE; ++u) x[u / 4][u & 3] = (float)vf[p][nt][u] * d[3][p * KG + col_token<DT>(g, u)];
          sp[nt] = split<3>(x, minus);
        }
        // four tiles of rows at a time, part by part: products that follow one another
        // add to different accumulators
#pragma unroll
        for (int kt0 = 0; kt0 < KT; kt0 += 4) {
          Frag f[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = col_frag<KPITCH>(sm.k + p * KG * KPITCH + kcol(kt0 + i), lane, KSTEP);
#pragma unroll
          for (int part = kParts<DT, 3> - 1; part >= 0; --part)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) S[kt0 + i][nt] = mma(f[i], sp[nt].part[part], S[kt0 + i][nt]);
        }
      }
    }
    __syncthreads();
    if constexpr (DOTS) {
      if (tid < CH) {
        const int t = t0 + (rev ? CH - 1 - tid : tid);
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) s += sm.dots[u][tid];
        if (t >= b && t < e) w.dots[(long)nh * w.T + t] = s;
      }
    }
  }
  float f = 1.0f;
  if (w.last_a0 && len > 0)
    f = exp2_parts(log2_decay(load_elem(w.gate, n * w.gs.n + h * w.gs.h, w.gate_f32), w.form));
  float* to = w.last ? w.last + nh * w.last_nh + seg * w.last_seg : nullptr;
  float* more = w.last2 ? w.last2 + nh * w.last2_nh : nullptr;
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    if (to) put_state(to, f);
    to = more;
  }
  if (w.decay) {
    total += __shfl_xor(total, 32);
    if (lane == 0) sm.totals[wave] = total;
    __syncthreads();
    if (tid == 0) {
      double sum = 0.0;
#pragma unroll
      for (int u = 0; u < WAVES; ++u) sum += sm.totals[u];
      w.decay[(long)nh * w.segs + seg] = power_of(sum);
    }
  }
}

// Columns of the state to a wave, in tiles of 16: blocks of four waves either way.
template <int VP> constexpr int kTilesOf = VP / 64;
template <int DT, int KP, int VP> using SmemOf = Smem<DT, KP, VP, kTilesOf<VP>>;

template <int DT, int KP, int VP, int MODE, bool VEC>
__global__ __launch_bounds__(256, KP == 64 && VP == 64 ? 3 : 2) void k_walk(Walk w) {
  extern __shared__ char smem[];
  walk<DT, KP, VP, kTilesOf<VP>, MODE, VEC>(w, blockIdx.x, smem);
}

// A walk with state [K][V] and one with [V][K], of `units` blocks each: of 16
// blocks in a row eight are the one's, on all XCDs, and eight the other's.
template <int DT, int KP, int VP, int MODE, int MODE2, bool VEC>
__global__ __launch_bounds__(256, KP == 64 && VP == 64 ? 3 : 2) void k_walk2(Walk w, Walk w2, int units) {
  extern __shared__ char smem[];
  const int unit = (int)(blockIdx.x >> 4) * 8 + (int)(blockIdx.x & 7);
  if (unit >= units) return;
  if ((blockIdx.x & 8) == 0) walk<DT, KP, VP, kTilesOf<VP>, MODE, VEC>(w, unit, smem);
  else walk<DT, VP, KP, kTilesOf<KP>, MODE2, VEC>(w2, unit, smem);
}

// Whole vectors, rows that do not overlap (a row past the last that exists is then
// past its end too), those of kAhead chunks within 2^30 bytes
// (kNoColumn less a chunk is past them).
template <int DT> bool vectors(const Walk& w) {
  constexpr int kVec = 16 / kBytes<DT>;
  auto fits = [](const Str& t, int len) {
    return len % kVec == 0 && (t.n | t.t | t.h) % kVec == 0 && t.t >= len && t.t < (1L << 30) / 4 / (kAhead * kChunk);
  };
  return (!w.y || fits(w.qs, w.K)) && fits(w.ks, w.K) && fits(w.vs, w.V) && (!w.y || fits(w.ys, w.V)) && (!w.x || fits(w.xs, w.V));
}

inline int mode_of(const Walk& w) { return !w.y ? kStates : w.x ? kOutDots : kOut; }

template <int DT, int KP, int VP>
hipError_t launch_walk_sized(const Walk& w, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((long)w.N * w.H * w.segs)), dim3(256), sizeof(SmemOf<DT, KP, VP>), s, w);
    return hipGetLastError();
  };
  const int mode = mode_of(w);
  if (vectors<DT>(w))
    return mode == kStates ? go(k_walk<DT, KP, VP, kStates, true>)
                           : mode == kOut ? go(k_walk<DT, KP, VP, kOut, true>) : go(k_walk<DT, KP, VP, kOutDots, true>);
  return mode == kStates ? go(k_walk<DT, KP, VP, kStates, false>)
                         : mode == kOut ? go(k_walk<DT, KP, VP, kOut, false>) : go(k_walk<DT, KP, VP, kOutDots, false>);
}

// w: outputs; w2: states or outputs.
template <int DT, int KP, int VP, bool VEC>
hipError_t launch_walk2_sized(const Walk& w, const Walk& w2, hipStream_t s) {
  const long units = (long)w.N * w.H * w.segs;
  auto go = [&](auto kernel) {
    constexpr size_t lds = sizeof(SmemOf<DT, KP, VP>) > sizeof(SmemOf<DT, VP, KP>) ? sizeof(SmemOf<DT, KP, VP>) : sizeof(SmemOf<DT, VP, KP>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((units + 7) / 8 * 16)), dim3(256), lds, s, w, w2, (int)units);
    return hipGetLastError();
  };
  if (mode_of(w2) == kStates) return w.x ? go(k_walk2<DT, KP, VP, kOutDots, kStates, VEC>) : go(k_walk2<DT, KP, VP, kOut, kStates, VEC>);
  return w.x ? go(k_walk2<DT, KP, VP, kOutDots, kOut, VEC>) : go(k_walk2<DT, KP, VP, kOut, kOut, VEC>);
}

template <int DT>
hipError_t launch_walk_dt(const Walk& w, const Walk* beside, hipStream_t s) {
  auto sized = [&](auto one, auto two) {   // the rounded sizes of K and V
    constexpr int KP = decltype(one)::value, VP = decltype(two)::value;
    if (!beside) return launch_walk_sized<DT, KP, VP>(w, s);
    return vectors<DT>(w) && vectors<DT>(*beside) ? launch_walk2_sized<DT, KP, VP, true>(w, *beside, s)
                                                   : launch_walk2_sized<DT, KP, VP, false>(w, *beside, s);
  };
  using A = std::integral_constant<int, 64>;
  using B = std::integral_constant<int, 128>;
  if (w.K <= 64) return w.V <= 64 ? sized(A{}, A{}) : sized(A{}, B{});
  return w.V <= 64 ? sized(B{}, A{}) : sized(B{}, B{});
}

}  // namespace
}  // namespace linattn
}  // namespace bc
