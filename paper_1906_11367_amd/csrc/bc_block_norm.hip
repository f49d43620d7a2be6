// The norms around a block, fused with its gate, residual sum and scale (gfx950).
// For every row of C channels:
//   p = norm(z) w_post within each of `groups` runs of channels (p = z without),
//   u = p act(gate),  r = x + scale u,  y = norm(r) w_pre,
// norm(v) = v rho, rho = (mean(v^2) + eps)^-1/2, of v less its mean for
// BC_NORM_LAYER.  The gradient to v through n = v rho, given dn, is
//   rho (dn - n mean(n dn) [- mean(dn)]).
// What bounds it: every tensor is read or written once, a few dozen operations
// an element, so memory.  A row stays in registers between its statistics: a team
// of lanes takes a row, 8 consecutive channels (16 bytes of bf16) a slot, no slot
// across two groups; rows of up to 64 slots (512 channels) share waves or take one,
// longer ones take a block.  The backward computes the forward's values again (in
// fp32, none read back rounded) and keeps each lane's share of the weights'
// gradients over all rows of its block; a second kernel sums the blocks in order.
// bf16: a norm with a gate of 16 heads of 128, 16384 rows: 44 us (201 MB, 4.6 TB/s),
// its gradients 88 (335 MB, 3.8); both norms with the residual sum of 8192 rows of
// 4096: 61 us (268 MB, 4.4 TB/s), the gradients 104 (403 MB, 3.9).  fp32, 777 rows of
// 3 x 279: 11 and 18 us, a row's chain of sums.  8 rows: 3.7 us, 7 us with the call.
// These are medians; single runs of the first two sizes' gradients are a seventh shorter.
// Where a variant stands beside another below, both ran in turn on one GPU.
#include <algorithm>

#include "bc_common.hpp"
#include "bc_internal.hpp"
#include "bc_scan.hpp"

namespace bc {
namespace {

using scan::kBF16;
using scan::kF32;
using scan::kBytes;
using scan::Raw;

struct Rows { const char* p; long stride; };   // of an input; null: none
struct OutRows { char* p; long stride; };

struct NormArgs {
  Rows z, gate, x;
  OutRows r, y;
  const float *w_post, *scale, *w_pre;
  Rows dr, dy;                  // backward
  OutRows dz, dgate, dx;
  float* part;                  // [blocks][2][C]: sums over rows of d n act(gate) and of dy norm(r); or null
  int wanted;                   // bit k: sum k is read
  int R, C, groups, size;       // size: channels of a group
  int per;                      // slots of a group
  int lanes;                    // of a team that shares its wave
  int mode;                     // how a group's slots are summed
  int layer, sigmoid, post, pre;
  float eps;
};

constexpr int kSumTeam = 0, kSumLanes = 1, kSumFew = 2, kSumShared = 3;
constexpr int kFew = 4;   // groups whose sums go side by side

// 1 / (1 + e^-g).  bf16: the exponential's argument is rounded once, which costs
// |g| 2^-24 of it; fp32: to a few units of 2^-24.
template <int DT> __device__ __forceinline__ float sigmoid(float g) {
  if constexpr (DT == kBF16) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.442695041f));
  const float e = expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e);
  return g >= 0.0f ? r : e * r;
}
// The same with its slope e / (1 + e)^2, e = e^-|g|: not s (1 - s), which has no digits
// left where s is close to 1.
template <int DT> __device__ __forceinline__ float sigmoid(float g, float& slope) {
  const float e = DT == kBF16 ? __builtin_amdgcn_exp2f(fabsf(g) * -1.442695041f) : expf(-fabsf(g));
  const float r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
  slope = er * r;
  return g >= 0.0f ? r : er;
}

// Sums over slots, by a team of W waves, or of `size` lanes of one (W = 1), NS
// slots a lane: slot i * size + lane.
template <int W, int NS> struct Team {
  static constexpr int kSlots = W == 1 ? 256 : 64 * W * NS;   // of a block, where they meet in LDS
  static constexpr int kRing = W > 1 ? 2 * 2 * kFew * W : 0;  // two places for the waves' sums
  static constexpr int kFloats = kRing + 4 * kSlots;
  float* lds;
  int lane, size;   // within the team; the team's lanes
  int base;         // the team's first slot of the block's
  int per, groups, mode;
  int turn = 0;

  template <int K> __device__ __forceinline__ void all(float (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = run_sum(v[k], W == 1 ? size : 64);
    if constexpr (W > 1) {
      // a place is written again after the next sum's barrier, when all have read it
      float* at = lds + turn * 2 * kFew * W;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) at[k * W + (threadIdx.x >> 6)] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) v[k] += at[k * W + w];
      }
    }
  }

  __device__ __forceinline__ int of(int i) const { return min((i * size + lane) / per, groups - 1); }   // slot i's group

  // over the whole row
  template <int K> __device__ __forceinline__ void row(float (&v)[NS][K]) {
    float s[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      s[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < NS; ++i) s[k] += v[i][k];
    }
    all<K>(s);
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int k = 0; k < K; ++k) v[i][k] = s[k];
  }

  // over each slot's group
  template <int K> __device__ __forceinline__ void group(float (&v)[NS][K]) {
    if (mode == kSumTeam) {
      row<K>(v);
    } else if (mode == kSumLanes) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int k = 0; k < K; ++k) v[i][k] = run_sum(v[i][k], per);
    } else if (mode == kSumFew) {
      float t[kFew * K];
#pragma unroll
      for (int f = 0; f < kFew; ++f)
#pragma unroll
        for (int k = 0; k < K; ++k) {
          t[f * K + k] = 0.0f;
#pragma unroll
          for (int i = 0; i < NS; ++i) t[f * K + k] += of(i) == f ? v[i][k] : 0.0f;
        }
      all<kFew * K>(t);
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int k = 0; k < K; ++k) {
          v[i][k] = t[k];
#pragma unroll
          for (int f = 1; f < kFew; ++f) v[i][k] = of(i) == f ? t[f * K + k] : v[i][k];
        }
    } else {
      float* slots = lds + kRing;
      float* sums = slots + 2 * kSlots;
      __syncthreads();   // the last sums have been read
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int k = 0; k < K; ++k) slots[k * kSlots + base + i * size + lane] = v[i][k];
      __syncthreads();
      // 8 lanes a group
      const int eight = lane >> 3, l = lane & 7;
      for (int g0 = 0; g0 < groups; g0 += size >> 3) {
        const int g = g0 + eight;
        float s[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
          s[k] = 0.0f;
          if (g < groups)
            for (int j = l; j < per; j += 8) s[k] += slots[k * kSlots + base + g * per + j];
          s[k] = run_sum(s[k], 8);
          if (g < groups && l == 0) sums[k * kSlots + base + g] = s[k];
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NS; ++i) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[i][k] = sums[k * kSlots + base + of(i)];
      }
    }
  }
};

// A lane's slots: 8 channels from col on, of which [lo, hi) are the slot's.  A
// group's last slot ends with the group and leaves to the one before what is that
// one's, so that every slot is read whole (groups below 8 channels: one slot, and
// its channels one by one).
template <int NS> struct Slots { int col[NS], lo[NS], hi[NS]; };

template <int DT> using Eight = Raw<scan::kWords<DT, 8>>;

template <int DT, int NS>
__device__ __forceinline__ void fetch(const Rows& t, long row, bool on, bool tiny, const Slots<NS>& s, Eight<DT> (&v)[NS]) {
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const char* p = t.p + (row * t.stride + s.col[i]) * kBytes<DT>;
    if (tiny) {
      v[i] = scan::load_vec<DT, 8>(p, on ? s.hi[i] : 0);
    } else {
      v[i] = {};
      if (on && s.hi[i] > 0) v[i] = scan::load_wide<DT, 8>(p);
    }
  }
}

template <int DT, int NS>
__device__ __forceinline__ void unpack(const Eight<DT> (&raw)[NS], bool whole, const Slots<NS>& s, float (&v)[NS][8]) {
#pragma unroll
  for (int i = 0; i < NS; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = scan::elem<DT, 8>(raw[i], e);
  if (!whole) {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = e >= s.lo[i] ? v[i][e] : 0.0f;
  }
}

// A row's values as they are stored, and the store of them.
template <int DT, int NS> struct Packed {
  Eight<DT> v[NS];
  __device__ __forceinline__ void set(const float (&x)[NS][8]) {
#pragma unroll
    for (int i = 0; i < NS; ++i) v[i] = scan::rounded<DT, 8>(x[i]);
  }
  __device__ __forceinline__ void store(const OutRows& t, long row, bool on, bool whole, const Slots<NS>& s) const {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      char* p = t.p + (row * t.stride + s.col[i]) * kBytes<DT>;
      if (!on || s.hi[i] == 0) continue;
      if (whole || (s.lo[i] == 0 && s.hi[i] == 8)) {
        *reinterpret_cast<scan::Loose<scan::kWords<DT, 8>, kBytes<DT>>*>(p) =
            __builtin_bit_cast(scan::Loose<scan::kWords<DT, 8>, kBytes<DT>>, v[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= s.lo[i] && e < s.hi[i]) {
            if constexpr (DT == kF32) reinterpret_cast<uint32_t*>(p)[e] = v[i][e];
            else reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(v[i][e / 2] >> (16 * (e & 1)));
          }
      }
    }
  }
};

template <int NS>
__device__ __forceinline__ void load_weights(const float* w, const Slots<NS>& s, float (&v)[NS][8]) {
#pragma unroll
  for (int i = 0; i < NS; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = w && e < s.hi[i] ? w[s.col[i] + e] : 1.0f;
}

// v -> v rho (less the mean), rho by slot.
template <bool kGroup, class Team, int NS>
__device__ __forceinline__ void normalise(Team& team, bool layer, float inv, float eps, const Slots<NS>& s,
                                          float (&v)[NS][8], float (&rho)[NS]) {
  float t[NS][1];
  auto sum = [&]() {
    if constexpr (kGroup) team.template group<1>(t);
    else team.template row<1>(t);
  };
  if (layer) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      t[i][0] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][0] += v[i][e];
    }
    sum();
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = e >= s.lo[i] && e < s.hi[i] ? v[i][e] - t[i][0] * inv : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    t[i][0] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[i][0] = fmaf(v[i][e], v[i][e], t[i][0]);
  }
  sum();
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    rho[i] = 1.0f / sqrtf(fmaf(t[i][0], inv, eps));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] *= rho[i];
  }
}

// dn (the gradient to n = norm(v)) -> the gradient to v.
template <bool kGroup, class Team, int NS>
__device__ __forceinline__ void norm_grad(Team& team, bool layer, float inv, const Slots<NS>& s, const float (&n)[NS][8],
                                          const float (&rho)[NS], float (&dn)[NS][8]) {
  if (!layer) {
    float t[NS][1];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      t[i][0] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][0] = fmaf(n[i][e], dn[i][e], t[i][0]);
    }
    if constexpr (kGroup) team.template group<1>(t);
    else team.template row<1>(t);
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) dn[i][e] = rho[i] * (dn[i][e] - n[i][e] * (t[i][0] * inv));
    return;
  }
  float t[NS][2];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    t[i][0] = t[i][1] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[i][0] = fmaf(n[i][e], dn[i][e], t[i][0]);
      t[i][1] += dn[i][e];
    }
  }
  if constexpr (kGroup) team.template group<2>(t);
  else team.template row<2>(t);
#pragma unroll
  for (int i = 0; i < NS; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      dn[i][e] = e >= s.lo[i] && e < s.hi[i] ? rho[i] * (dn[i][e] - t[i][1] * inv - n[i][e] * (t[i][0] * inv)) : 0.0f;
}

// Blocks of the forward: as many as the card holds at once, each with a run of rows
// (its weights are loaded once, and the next row's inputs ahead).  8192 rows of
// 4096 bf16 with residual and both norms: 58 us, with 2048 blocks 76.
constexpr int fwd_blocks(int W) { return W <= 2 ? 2048 : W == 4 ? 1536 : W == 8 ? 768 : 256; }

// Waves a SIMD: what the registers of the variant allow without a spill (a reload
// waits for the loads ahead too).
constexpr int waves_of(int dt, int W, int NS, bool bwd, bool both) {
  if (W == 16) return 4;
  if (NS == 2) return 2;
  if (bwd) return dt == kBF16 && !both ? 4 : 2;
  return dt == kBF16 ? (both ? 5 : 6) : 4;
}

// GATE, PRE: there is a gate; there is a y (or its gradient).
template <int DT, int W, int NS, bool BWD, bool GATE, bool PRE>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, waves_of(DT, W, NS, BWD, GATE && PRE)) void k_block_norm(NormArgs a) {
  using T = Team<W, NS>;
  __shared__ float lds[T::kFloats];
  const int tid = threadIdx.x;
  T team;
  team.lds = lds;
  team.size = W == 1 ? a.lanes : 64 * W;
  team.lane = W == 1 ? tid & (a.lanes - 1) : tid;
  const int which = W == 1 ? tid / a.lanes : 0, teams = W == 1 ? 256 / a.lanes : 1;
  team.base = which * team.size;
  team.per = a.per;
  team.groups = max(a.groups, 1);
  team.mode = a.mode;
  const bool tiny = a.size < 8, whole = a.size % 8 == 0;

  Slots<NS> s;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int j = i * team.size + team.lane, g = j / a.per, k = j % a.per;
    const int over = tiny ? 0 : max(k * 8 + 8 - a.size, 0);   // past the group's end
    s.col[i] = g < team.groups ? g * a.size + k * 8 - over : 0;
    s.lo[i] = over;
    s.hi[i] = g < team.groups ? min(a.size, 8) : 0;
  }
  float w[NS][8], w_pre[NS][8];   // w_post scale, w_pre
  {
    float scale[NS][8];
    load_weights<NS>(a.w_post, s, w);
    load_weights<NS>(a.scale, s, scale);
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[i][e] *= scale[i][e];
  }
  if constexpr (PRE) load_weights<NS>(a.w_pre, s, w_pre);
  const float inv_group = 1.0f / (float)a.size, inv_row = 1.0f / (float)a.C;

  float sum[2][NS][8];
  if constexpr (BWD) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[k][i][e] = 0.0f;
  }

  // a row's inputs are on their way while the row before it is worked on, where the
  // registers hold them
  constexpr bool AHEAD = NS == 1 ? W < 16 || !(BWD && PRE) : W < 16 && (!PRE || (!GATE && DT == kBF16));
  constexpr bool X = PRE || !BWD;   // x is read
  Eight<DT> rz[NS], rg[NS], rx[NS], rdr[NS], rdy[NS];
  auto get = [&](long row0) {
    const long row = row0 + which;
    const bool on = row < a.R;
    fetch<DT, NS>(a.z, row, on, tiny, s, rz);
    if constexpr (GATE) fetch<DT, NS>(a.gate, row, on, tiny, s, rg);
    if constexpr (X) fetch<DT, NS>(a.x, row, on && a.x.p, tiny, s, rx);
    if constexpr (BWD) fetch<DT, NS>(a.dr, row, on && a.dr.p, tiny, s, rdr);
    if constexpr (BWD && PRE) fetch<DT, NS>(a.dy, row, on, tiny, s, rdy);
  };
  const long step = (long)gridDim.x * teams;
  long row0 = (long)blockIdx.x * teams;
  if (AHEAD && row0 < a.R) get(row0);
  for (; row0 < a.R; row0 += step) {
    const long row = row0 + which;
    const bool on = row < a.R;
    if constexpr (!AHEAD) get(row0);
    float n[NS][8], g[NS][8], r[NS][8], d[NS][8], dy[NS][8], rho1[NS], rho2[NS];
    unpack<DT, NS>(rz, whole, s, n);
    if constexpr (GATE) unpack<DT, NS>(rg, whole, s, g);
    if constexpr (X) unpack<DT, NS>(rx, whole, s, r);
    if constexpr (BWD) unpack<DT, NS>(rdr, whole, s, d);
    if constexpr (BWD && PRE) unpack<DT, NS>(rdy, whole, s, dy);
    if (AHEAD && row0 + step < a.R) get(row0 + step);
    if (a.post) normalise<true>(team, a.layer, inv_group, a.eps, s, n, rho1);
    float phi[NS][8];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (GATE) {
          float sg, slope;
          if constexpr (BWD) sg = sigmoid<DT>(g[i][e], slope);
          else sg = sigmoid<DT>(g[i][e]);
          phi[i][e] = a.sigmoid ? sg : g[i][e] * sg;
          if constexpr (BWD) g[i][e] = a.sigmoid ? slope : fmaf(g[i][e], slope, sg);   // phi's slope
        }
        if constexpr (X) r[i][e] = fmaf(GATE ? n[i][e] * phi[i][e] : n[i][e], w[i][e], r[i][e]);
      }
    // what goes to memory is kept until the row's end: the next row's loads are
    // waited for before any store is on its way, since such waits count both
    Packed<DT, NS> o[3];
    if constexpr (!BWD) {
      o[0].set(r);
      if constexpr (PRE) {
        normalise<false>(team, a.layer, inv_row, a.eps, s, r, rho2);
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) r[i][e] *= w_pre[i][e];
        o[1].set(r);
      }
    } else {
      if constexpr (PRE) {
        normalise<false>(team, a.layer, inv_row, a.eps, s, r, rho2);
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sum[1][i][e] = fmaf(dy[i][e], r[i][e], sum[1][i][e]);
            dy[i][e] *= w_pre[i][e];
          }
        norm_grad<false>(team, a.layer, inv_row, s, r, rho2, dy);
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) d[i][e] += dy[i][e];
      }
      o[0].set(d);
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (GATE) {
            g[i][e] *= d[i][e] * w[i][e] * n[i][e];
            d[i][e] *= phi[i][e];
          }
          sum[0][i][e] = fmaf(d[i][e], n[i][e], sum[0][i][e]);
          d[i][e] *= w[i][e];
        }
      if constexpr (GATE) o[1].set(g);
      if (a.dz.p) {
        if (a.post) norm_grad<true>(team, a.layer, inv_group, s, n, rho1, d);
        o[2].set(d);
      }
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        asm volatile("" : "+v"(rz[i]));
        if constexpr (GATE) asm volatile("" : "+v"(rg[i]));
        if constexpr (X) asm volatile("" : "+v"(rx[i]));
        if constexpr (BWD) asm volatile("" : "+v"(rdr[i]));
        if constexpr (BWD && PRE) asm volatile("" : "+v"(rdy[i]));
      }
    }
    if constexpr (!BWD) {
      if (a.r.p) o[0].store(a.r, row, on, whole, s);
      if constexpr (PRE) o[1].store(a.y, row, on, whole, s);
    } else {
      if (a.dx.p) o[0].store(a.dx, row, on, whole, s);
      if constexpr (GATE)
        if (a.dgate.p) o[1].store(a.dgate, row, on, whole, s);
      if (a.dz.p) o[2].store(a.dz, row, on, whole, s);
    }
  }
  if constexpr (BWD) {
    if (a.part) {
      float* out = a.part + (long)blockIdx.x * 2 * a.C;
      // teams of one block: in order, through LDS
      if (W == 1 && teams > 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (!(a.wanted >> k & 1)) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __syncthreads();
            lds[tid] = sum[k][0][e];
            __syncthreads();
            if (which == 0) {
              float t = 0.0f;
              for (int u = 0; u < teams; ++u) t += lds[u * team.size + team.lane];
              if (e >= s.lo[0] && e < s.hi[0]) out[(long)k * a.C + s.col[0] + e] = t;
            }
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (a.wanted >> k & 1)
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= s.lo[i] && e < s.hi[i]) out[(long)k * a.C + s.col[i] + e] = sum[k][i][e];
      }
    }
  }
}

// Blocks of the backward, and shares of the weights' gradients: 2048 waves or more, or
// one block a CU where it holds no more.
// With both norms and the weights' gradients, bf16, 65536 rows of 640 (blocks of two
// waves): 150 us, with 512 blocks 293; 8192 rows of 4096: 98, with 1024 blocks 110.
constexpr int part_blocks(int W) { return W == 2 ? 1024 : W == 16 ? 256 : 512; }
// Rows a block takes at least, past kFewBlocks blocks: a share costs more than a row or
// two.  600 rows of 4096: 27 us, a block a row 32 to 41; 300 rows of 1024: 12.1, 12.8.
// Fewer rows follow one another for nothing: 11 rows of 5272 in 11 blocks 21 us, in 3 30.
constexpr int part_rows(int W) { return W == 1 ? 1 : W < 8 ? 2 : 4; }
constexpr long kFewBlocks = 128;

// The weights' gradients from the blocks' sums part [P][2][C], 32 channels a block,
// a lane of 32 the blocks p, p + 32, ..., all on their way at once (16 MB of 512 x 4096 in
// 5 us).  With A the sum of d n act(gate), the gradient to w_post is scale A and that to
// scale w_post A.
struct WeightGrads {
  const float *part, *w_post, *scale;
  float *dw_post, *dscale, *dw_pre;
  int P, C;
};
template <int BLOCKS> __global__ __launch_bounds__(1024) void k_norm_weights(WeightGrads a) {
  __shared__ float lds[32][33];
  const int blocks = (a.C + 31) / 32, k = blockIdx.x / blocks, col = threadIdx.x & 31, row = threadIdx.x >> 5;
  const int c = min((int)(blockIdx.x % blocks) * 32 + col, a.C - 1);
  if (k == 0 ? !a.dw_post && !a.dscale : !a.dw_pre) return;
  float v[BLOCKS / 32], s = 0.0f;
#pragma unroll
  for (int i = 0; i < BLOCKS / 32; ++i) v[i] = a.part[((long)min(row + 32 * i, a.P - 1) * 2 + k) * a.C + c];
#pragma unroll
  for (int i = 0; i < BLOCKS / 32; ++i) s += row + 32 * i < a.P ? v[i] : 0.0f;
  lds[col][row] = s;
  __syncthreads();
  // 32 lanes a channel
  const float t = run_sum(lds[row][col], 32);
  const int to = (int)(blockIdx.x % blocks) * 32 + row;
  if (col != 0 || to >= a.C) return;
  if (k == 1) {
    a.dw_pre[to] = t;
  } else {
    if (a.dw_post) a.dw_post[to] = a.scale ? t * a.scale[to] : t;
    if (a.dscale) a.dscale[to] = a.w_post ? t * a.w_post[to] : t;
  }
}

inline int slots_of(int C, int groups) {
  const int G = std::max(groups, 1);
  return G * ((C / G + 7) / 8);
}

template <int DT, bool BWD, bool GATE, bool PRE>
hipError_t launch_norm(NormArgs& a, int* blocks, hipStream_t s) {
  const int slots = slots_of(a.C, a.groups);
  const int G = std::max(a.groups, 1);
  a.size = a.C / G;
  a.per = slots / G;
  a.lanes = 64;
  const bool pow2 = (a.per & (a.per - 1)) == 0 && a.per <= 64;
  auto go = [&](auto kernel, int threads, int teams, int W) {
    long want = ((long)a.R + teams - 1) / teams;
    if (BWD) want = std::max((want + part_rows(W) - 1) / part_rows(W), std::min(want, kFewBlocks));
    *blocks = (int)std::min<long>(want, BWD ? part_blocks(W) : fwd_blocks(W));
    a.mode = G == 1 ? kSumTeam : pow2 ? kSumLanes : G <= kFew ? kSumFew : kSumShared;
    hipLaunchKernelGGL(kernel, dim3((unsigned)*blocks), dim3((unsigned)threads), 0, s, a);
    return hipGetLastError();
  };
  if (slots <= 64) {
    a.lanes = 8;
    while (a.lanes < slots) a.lanes *= 2;
    return go(k_block_norm<DT, 1, 1, BWD, GATE, PRE>, 256, 256 / a.lanes, 1);
  }
  if (slots <= 128) return go(k_block_norm<DT, 2, 1, BWD, GATE, PRE>, 128, 1, 2);
  if (slots <= 256) return go(k_block_norm<DT, 4, 1, BWD, GATE, PRE>, 256, 1, 4);
  if (slots <= 512) return go(k_block_norm<DT, 8, 1, BWD, GATE, PRE>, 512, 1, 8);
  if (slots <= 1024) {
    // 8 waves with 256 registers each have room to read ahead: 4096 rows of 8192 bf16,
    // both norms, 99 us; 16 waves 131
    if constexpr (BWD) return go(k_block_norm<DT, 8, 2, BWD, GATE, PRE>, 512, 1, 16);
    else return go(k_block_norm<DT, 16, 1, BWD, GATE, PRE>, 1024, 1, 16);
  }
  return go(k_block_norm<DT, 16, 2, BWD, GATE, PRE>, 1024, 1, 16);
}

template <int DT, bool BWD>
hipError_t launch_norm(NormArgs& a, int* blocks, hipStream_t s) {
  if (a.gate.p) return a.pre ? launch_norm<DT, BWD, true, true>(a, blocks, s) : launch_norm<DT, BWD, true, false>(a, blocks, s);
  return a.pre ? launch_norm<DT, BWD, false, true>(a, blocks, s) : launch_norm<DT, BWD, false, false>(a, blocks, s);
}

}  // namespace

bool block_norm_takes(int C, int groups) { return slots_of(C, groups) <= 2048; }

size_t block_norm_workspace_bytes(int R, int C) { return (size_t)std::min(R, C <= 1024 ? part_blocks(2) : part_blocks(4)) * 2 * C * 4; }

static Rows rows(const NormRows& t) { return {static_cast<const char*>(t.p), t.stride}; }
static OutRows out_rows(const NormRows& t) { return {static_cast<char*>(const_cast<void*>(t.p)), t.stride}; }

hipError_t launch_block_norm(const BlockNorm& b, bool bwd, hipStream_t s) {
  NormArgs a{};
  a.z = rows(b.z);
  a.gate = rows(b.gate);
  a.x = rows(b.x);
  a.r = out_rows(b.r);
  a.y = out_rows(b.y);
  a.w_post = b.w_post;
  a.scale = b.scale;
  a.w_pre = b.w_pre;
  a.dr = rows(b.dr);
  a.dy = rows(b.dy);
  a.dz = out_rows(b.dz);
  a.dgate = out_rows(b.dgate);
  a.dx = out_rows(b.dx);
  a.R = b.R;
  a.C = b.C;
  a.groups = b.groups;
  a.layer = b.layer;
  a.sigmoid = b.sigmoid;
  a.post = b.groups > 0;
  a.pre = bwd ? b.dy.p != nullptr : b.y.p != nullptr;
  a.eps = b.eps;
  int blocks = 0;
  if (!bwd) return b.dt == kBF16 ? launch_norm<kBF16, false>(a, &blocks, s) : launch_norm<kF32, false>(a, &blocks, s);
  const bool weights = b.dw_post || b.dscale || b.dw_pre;
  a.part = weights ? static_cast<float*>(b.ws) : nullptr;
  a.wanted = (b.dw_post || b.dscale ? 1 : 0) | (b.dw_pre ? 2 : 0);
  const hipError_t e = b.dt == kBF16 ? launch_norm<kBF16, true>(a, &blocks, s) : launch_norm<kF32, true>(a, &blocks, s);
  if (e != hipSuccess || !weights) return e;
  const WeightGrads w{a.part, b.w_post, b.scale, b.dw_post, b.dscale, b.dw_pre, blocks, b.C};
  hipLaunchKernelGGL(blocks > 512 ? k_norm_weights<1024> : k_norm_weights<512>, dim3((unsigned)(2 * ((b.C + 31) / 32))), dim3(1024), 0, s, w);
  return hipGetLastError();
}

}  // namespace bc
