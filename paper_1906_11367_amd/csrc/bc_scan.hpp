// Shared device code of the gated scan (gfx950).
//
// The recurrence h_t = a_t h_{t-1} + b_t composes: a run of steps takes the
// state h before it to A h + B, and the run (A, B) followed by (A', B') is
// (A' A, A' B + B').  A tile of steps is cut into short runs, one per lane,
// whose pairs are scanned across the lanes and waves; each lane then walks its
// run from the state before it.  The backward is the same recurrence with time
// reversed: with r_t the gradient carried to the state before step t,
//   delta_t = grad_y_t + r_{t+1},  r_t = a_t delta_t = a_t r_{t+1} + a_t grad_y_t,
// and the coefficient's gradient needs h_{t-1}, which is computed again from
// states the forward kept (one every 128 steps of tokens, every 256 of fp32 maps and
// 512 of bf16 ones) rather than read from the rounded outputs.
// States, coefficients and gradients are fp32 throughout; bf16 is storage only,
// rounded once, to nearest even.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "bc_internal.hpp"

namespace bc {
namespace scan {

constexpr int kF32 = 1, kBF16 = 2;      // storage codes, as bc_dtype
constexpr int kLogit = 0, kValue = 1;   // gate forms, as bc_gate_form

template <int DT> constexpr int kBytes = DT == kBF16 ? 2 : 4;

template <int N> using Raw = uint32_t __attribute__((ext_vector_type(N)));
template <int DT, int V> constexpr int kWords = V * kBytes<DT> / 4;

// Element alignment is all a row has (a row of odd length, or a slice of one):
// one wide access at that alignment, which global memory allows here.
template <int N, int kAlign> struct __attribute__((packed, aligned(kAlign))) Loose { uint32_t w[N]; };

// V elements from p.
template <int DT, int V>
__device__ __forceinline__ Raw<kWords<DT, V>> load_wide(const char* p) {
  return __builtin_bit_cast(Raw<kWords<DT, V>>, *reinterpret_cast<const Loose<kWords<DT, V>, kBytes<DT>>*>(p));
}

// V elements from p, of which the first `avail` exist (the rest read as zero).
// Loads that are to be in flight together do not come through here: the short
// form writes the registers of the wide one, which first has to arrive.  They
// are load_wide in a branch that all lanes of the block take.
template <int DT, int V>
__device__ __forceinline__ Raw<kWords<DT, V>> load_vec(const char* p, int avail) {
  constexpr int W = kWords<DT, V>;
  Raw<W> r;
  if (avail >= V) {
    r = load_wide<DT, V>(p);
  } else {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if constexpr (DT == kBF16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
        const uint32_t lo = 2 * k < avail ? q[2 * k] : 0u, hi = 2 * k + 1 < avail ? q[2 * k + 1] : 0u;
        r[k] = lo | (hi << 16);
      } else {
        r[k] = k < avail ? reinterpret_cast<const uint32_t*>(p)[k] : 0u;
      }
    }
  }
  return r;
}

template <int DT, int V>
__device__ __forceinline__ float elem(const Raw<kWords<DT, V>>& r, int k) {
  if constexpr (DT == kBF16) return __uint_as_float((k & 1) ? r[k / 2] & 0xffff0000u : r[k / 2] << 16);
  else return __uint_as_float(r[k]);
}

// Two values to a bf16 pair, nearest even (one instruction here).
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
  const __bf16 a = (__bf16)lo, b = (__bf16)hi;
  return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
}

template <int DT, int V>
__device__ __forceinline__ Raw<kWords<DT, V>> rounded(const float (&v)[V]) {
  Raw<kWords<DT, V>> r;
#pragma unroll
  for (int k = 0; k < kWords<DT, V>; ++k) {
    if constexpr (DT == kBF16) r[k] = pair_bf16(v[2 * k], v[2 * k + 1]);
    else r[k] = __float_as_uint(v[k]);
  }
  return r;
}

// stream: past the caches (see streams()).
template <int DT, int V>
__device__ __forceinline__ void store_wide(char* p, const float (&v)[V], bool stream) {
  constexpr int W = kWords<DT, V>;
  const Raw<W> r = rounded<DT, V>(v);
  if (stream) {
    typedef Raw<W> Any __attribute__((aligned(kBytes<DT>)));
    asm volatile("");   // keeps the compiler from merging the two stores into a plain one
    __builtin_nontemporal_store(r, reinterpret_cast<Any*>(p));
    asm volatile("");
  } else {
    *reinterpret_cast<Loose<W, kBytes<DT>>*>(p) = __builtin_bit_cast(Loose<W, kBytes<DT>>, r);
  }
}

template <int DT, int V>
__device__ __forceinline__ void store_vec(char* p, int avail, const float (&v)[V]) {
  constexpr int W = kWords<DT, V>;
  const Raw<W> r = rounded<DT, V>(v);
  if (avail >= V) {
    *reinterpret_cast<Loose<W, kBytes<DT>>*>(p) = __builtin_bit_cast(Loose<W, kBytes<DT>>, r);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (k >= avail) break;
      if constexpr (DT == kBF16) reinterpret_cast<uint16_t*>(p)[k] = (uint16_t)(r[k / 2] >> (16 * (k & 1)));
      else reinterpret_cast<uint32_t*>(p)[k] = r[k];
    }
  }
}

template <int DT, int V>
__device__ __forceinline__ void store_zero(char* p, int avail) {
  const float z[V] = {};
  store_vec<DT, V>(p, avail, z);
}

// Gates of steps past a sequence's end: a = 1 exactly (and c = 0 in the logit
// form; the input reads as zero there), so that the state stays as it is.
template <int DT, int FORM, int V>
__device__ __forceinline__ Raw<kWords<DT, V>> hold_gate() {
  constexpr uint32_t bits = FORM == kValue ? 0x3f800000u : 0x7f800000u;   // 1, or infinity
  Raw<kWords<DT, V>> r;
#pragma unroll
  for (int k = 0; k < kWords<DT, V>; ++k) r[k] = DT == kBF16 ? bits | bits >> 16 : bits;
  return r;
}

// exp(-v), v >= 0.  fp32 storage: the rounding of v / ln 2, which would grow
// with v, is put back to first order; 3 units of 2^-24 are left, of the exponential
// (an ulp) and the last product.  bf16 storage, whose gates are off by 2^-9 of
// themselves already, leaves it: 1.22 v units more.
template <int DT>
__device__ __forceinline__ float exp_neg(float v) {
  const float t = v * -1.44269504f;
  const float e = __builtin_amdgcn_exp2f(t);
  if constexpr (DT == kBF16) return e;
  const float lo = __fmaf_rn(v, -1.44269504f, -t) + v * -1.92596299e-8f;
  return v < 128.f ? __fmaf_rn(e, lo * 0.693147181f, e) : e;   // 0 there already (and at infinity)
}

// Coefficient a of the state and c of the input.  The logit form takes both
// from exp(-|gate|), so that neither a nor 1 - a loses its digits where it is
// small: 4 units more, of the sum, the reciprocal (an ulp) and the product.
// gate = -infinity is an exact reset (a = 0, c = 1).
template <int DT, int FORM>
__device__ __forceinline__ void coefficients(float gate, float& a, float& c) {
  if constexpr (FORM == kValue) {
    a = gate;
    c = 1.f;
  } else {
    const float e = exp_neg<DT>(fabsf(gate));
    const float r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
    a = gate >= 0.f ? r : er;
    c = gate >= 0.f ? er : r;   // a NaN is in r and er already
  }
}

// c x, the input's share of a step.
template <int FORM>
__device__ __forceinline__ float input_share(float c, float x) { return FORM == kValue ? x : c * x; }

struct FwdArgs {
  const char *gate, *x;
  long bs, rs;              // batch and row strides of gate and x, in elements
  const float* h0;          // [N][C] or null
  const int* lengths;       // [N] or null
  char* y;                  // dense
  float* h_last;            // [N][C] or null
  float* states;            // or null
  int N, T, C;
  int slabs, tiles, groups;   // tokens: channel slabs, tiles of time steps, groups of tiles
  bool stream;              // y past the caches
  unsigned long long *tickets, *agg, *pre;   // chained: see bc_scan.hip
};

struct BwdArgs {
  const char *gate, *x;
  long bs, rs;
  const float* states;
  const int* lengths;
  const char* gy;           // dense
  const float* gh_last;     // [N][C] or null
  char *ggate, *gx;
  long gbs, grs;            // strides of ggate and gx
  float* gh0;               // [N][C] or null
  int N, T, C;
  int slabs, tiles, groups;
  bool stream;              // ggate and gx past the caches
  unsigned long long *tickets, *agg, *pre;
};

__device__ __forceinline__ int seq_len(const int* lengths, int n, int T) {
  return lengths ? max(0, min(lengths[n], T)) : T;
}

// Outputs of `elements` in rows of `rs` go past the caches where they are
// larger than the XCDs' L2 and their rows are whole runs of `run` bytes: 64 where
// a row is written in parts, which would each cost a read of a line that they
// share; 16, a lane's piece, where a wave writes 1 KiB of a row in one piece.
// Measured with and without, us: forward 1 x 65536 x 1024 bf16 94 and 103, backward
// 8 x 4096 x 2048 bf16 156 and 165, mix 16000 x 1024 to 4704 bf16 107 and 110;
// rows of 837 fp32 32 and 24, of 1032 bf16 64 and 57; maps 32 x 512 x 4096 bf16 68
// and 82, 32 x 256 x 4104 bf16 47 and 53.
inline bool streams(double elements, long rs, int dt, const void* a, const void* b, int run) {
  const int e = dt == kBF16 ? 2 : 4;
  return elements * e >= 32e6 && rs * e % run == 0 && ((uintptr_t)a | (uintptr_t)b) % run == 0;
}

}  // namespace scan
}  // namespace bc
