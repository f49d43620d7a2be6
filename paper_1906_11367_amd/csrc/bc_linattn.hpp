// Linear attention with a decay for each head (gfx950): shared device code.
//
// For a sequence and head, from S_{-1} = s0,
//   S_t = a_t S_{t-1} + k_t v_t^T,   y_t = scale S_t^T q_t.
// In chunks of tokens, with L_i the sum of log a over the chunk up to i, what
// token j leaves reaches token i >= j by exp(L_i - L_j):
//   y_i = scale (sum_{j <= i} exp(L_i - L_j) (q_i . k_j) v_j + exp(L_i) S^T q_i),
//   S' = exp(L_end) S + sum_j exp(L_end - L_j) k_j v_j^T,
// four matrix products with S held in registers from chunk to chunk.  All the
// exponents are sums of log a: there is no division by a decay, decays up to one
// cannot overflow, and a reset (a = 0) is exact.  Decays above one multiply before
// they meet a state, so the products of a chunk's have to stay inside fp32's range
// (those of a segment's need not: Power).
//
// The gradients are the same walk over other operands.  With R_t the gradient
// to S_t, R_t = scale q_t dy_t^T + a_{t+1} R_{t+1}:
//   dq_t = scale S_t dy_t : the walk forward with (q, k, v) = (dy, v, k), state S^T;
//   dv_t = R_t^T k_t      : backward in time with (k, q, dy), state R, a shifted;
//   dk_t = R_t v_t        : backward in time with (v, dy, q), state R^T;
// and, as every path from a token before t to one at or after it passes a_t,
//   d/d(log a_t) = sum_{s >= t} (q_s . dq_s - k_s . dk_s) + <S_end, R_end>,
// the sum within a span of tokens, the last term over its end.
#pragma once
#include "bc_scan.hpp"

namespace bc {
namespace linattn {

using scan::kBF16;
using scan::kF32;
using scan::kBytes;
using scan::Raw;

constexpr int kGateLogit = 0, kGateLog = 2;   // as bc_gate_form

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
#define BC_LDS __attribute__((address_space(3)))

struct Str { long n, t, h; };   // elements between batches, tokens, heads

// A logarithm of a decay below this leaves nothing of a state (as -infinity).
constexpr float kLogMin = -1.0e4f;
constexpr double kLog2e = 1.4426950408889634;

// log2 of the decay, from the gate.
__device__ __forceinline__ double log2_decay(float g, int form) {
  float v = g;
  if (form == kGateLogit) v = fminf(g, 0.0f) - log1pf(expf(-fabsf(g)));
  if (v < kLogMin) v = kLogMin;   // (a NaN stays one)
  return (double)v * kLog2e;
}

__device__ __forceinline__ float load_elem(const char* p, long i, bool f32) {
  if (f32) return reinterpret_cast<const float*>(p)[i];
  return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
}

// 2^(hi + lo), |lo| <= ulp(hi).
__device__ __forceinline__ float exp2_parts(double x) {
  const float hi = (float)x, e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, (float)(x - (double)hi) * 0.6931472f, e);
}

// 2^x as two factors that are finite, the first a power of two: s 2^x leaves fp32's
// range only where the product does.
struct Power { float a, b; };
__device__ __forceinline__ Power power_of(double x) {
  const double c = x < -1000.0 ? -1000.0 : x > 250.0 ? 250.0 : x;   // (a NaN stays one; -1000: zero)
  const double half = __builtin_rint(c * 0.5);
  return {__builtin_amdgcn_exp2f((float)half), exp2_parts(c - half)};
}
// s 2^x + add
__device__ __forceinline__ float scaled(float s, const Power& p, float add) { return fmaf(s * p.a, p.b, add); }

// The walk of one block over a segment of one sequence and head: operands are
// named as in the forward.
struct Walk {
  const char *q, *k, *v, *gate;
  Str qs, ks, vs, gs;
  int qd, kd, vd;            // head h reads head h / qd of q, ...
  int K, V;                  // lengths of q's and k's rows, of v's and y's
  int gate_f32, form;
  const int* lengths;
  int N, T, H;
  int rev;                   // backward in time, with the decay of the token after
  int seg, segs;             // tokens of a segment (whole chunks), segments
  const float* init;         // state before a segment, or null: zero
  long init_nh, init_seg;
  float* first;              // the initial state once more (one segment), entries last2_nh apart
  int rows_first;            // states in memory are [K][V]; else [V][K]
  float* last;               // state after a segment, or null
  long last_nh, last_seg;
  float* last2;              // the same once more (one segment), entries last2_nh apart
  long last2_nh;
  int last_a0;               // rev: `last` is times the first token's decay
  Power* decay;              // [nh][segs]: the segments' decays, or null
  char* y;                   // null: states only
  Str ys;
  int y_f32;
  float scale;               // of y
  float kv;                  // of every k v^T
  const char* x;             // dots[nh][t] = x_t . y_t, or null
  Str xs;
  int xd;
  float* dots;
};

constexpr int kChunk = 32;   // tokens of a chunk

// Walks of their own, or two over the same segments in one launch, block beside
// block on one XCD: what both read is fetched once.
hipError_t launch_walk_bf16(const Walk& w, const Walk* beside, hipStream_t s);
hipError_t launch_walk_f32(const Walk& w, const Walk* beside, hipStream_t s);

}  // namespace linattn
}  // namespace bc
