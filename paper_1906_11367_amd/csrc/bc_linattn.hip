// Linear attention with a decay for each head: how a call is divided, the joints
// between segments, the gates' gradients, and the step for single tokens.  The
// walk over segments is bc_linattn_walk.hpp's.
#include <algorithm>

#include "bc_internal.hpp"
#include "bc_linattn.hpp"

namespace bc {
namespace linattn {
namespace {

// States at the segments' borders from what the segments leave by themselves, in
// place: entry i is border i; forward, entry s + 1 holds segment s's own state, and
// the states follow from the first border on; backward in time, entry s, from the
// last.  A thread a cell, its chain's entries read eight at a time.  Bound by memory:
// 64 heads of 128 x 128, 8 segments, 34 MB in and out in 16 us (4.2 TB/s).
struct Joint {
  float* entry;
  long entry_nh;           // (segs + 1) cells
  const float* start;      // [nh][cells], or null: zero
  const Power* decay;      // [nh][segs]
  float* last;             // [nh][cells], or null
  const char* gate;        // rev: last is times the first token's decay
  Str gs;
  int gate_f32, form;
  const int* lengths;
  int H, segs, cells, rev;
};

constexpr int kJointAhead = 8;   // segments whose entries are on their way

__global__ __launch_bounds__(256) void k_join(Joint j) {
  const int blocks = (j.cells + 255) / 256, nh = blockIdx.x / blocks, cell = blockIdx.x % blocks * 256 + threadIdx.x;
  if (cell >= j.cells) return;
  float* p = j.entry + nh * j.entry_nh + cell;
  const Power* dec = j.decay + (long)nh * j.segs;
  float s = j.start ? j.start[(long)nh * j.cells + cell] : 0.0f;
  p[j.rev ? (long)j.segs * j.cells : 0] = s;
  auto at = [&](int i) { return (long)(j.rev ? j.segs - 1 - i : i + 1) * j.cells; };
  for (int i0 = 0; i0 < j.segs; i0 += kJointAhead) {
    float add[kJointAhead];
    Power d[kJointAhead];
#pragma unroll
    for (int u = 0; u < kJointAhead; ++u) {
      const int i = min(i0 + u, j.segs - 1);
      add[u] = p[at(i)];
      d[u] = dec[j.rev ? j.segs - 1 - i : i];
    }
#pragma unroll
    for (int u = 0; u < kJointAhead; ++u) {
      if (i0 + u < j.segs) {
        s = scaled(s, d[u], add[u]);
        p[at(i0 + u)] = s;
      }
    }
  }
  if (j.last) {
    const int n = nh / j.H, h = nh % j.H;
    float f = 1.0f;
    if (j.rev && (!j.lengths || j.lengths[n] > 0))
      f = exp2_parts(log2_decay(load_elem(j.gate, n * j.gs.n + h * j.gs.h, j.gate_f32), j.form));
    j.last[(long)nh * j.cells + cell] = s * f;
  }
}

// The gates' gradients of one segment: the sum of q . dq - k . dk from a token to
// the segment's end, and what crosses that end, <state, gradient> of the border.  A
// block a segment; the sums are fp64 (they are differences of large numbers).  Bound
// by the states' bytes: 64 heads of 128 x 128, 8 segments, 71 MB in 22 us (3.2 TB/s).
struct GateGrad {
  const float *dq, *dk;          // [nh][T]: q_t . dq_t, k_t . dk_t
  const float* state;            // after segment s: at nh * state_nh + (s + 1) cells
  long state_nh;
  const float* grad;             // its gradient, before the next token's decay; null: zero
  long grad_nh, grad_seg;
  const char* gate;
  Str gs;
  int gate_f32, form;
  char* out;
  Str os;
  const int* lengths;
  int T, H, seg, segs, cells;
};

__global__ __launch_bounds__(256) void k_gate_grad(GateGrad a) {
  __shared__ double part[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sp = blockIdx.x % a.segs, nh = blockIdx.x / a.segs, n = nh / a.H, h = nh % a.H;
  const int len = a.lengths ? min(max(a.lengths[n], 0), a.T) : a.T;
  const int b = sp * a.seg, e = min(b + a.seg, a.T);
  const long g0 = n * a.gs.n + h * a.gs.h;
  double carry = 0.0;
  if (a.grad && b < len) {
    const float* x = a.state + nh * a.state_nh + (long)(sp + 1) * a.cells;
    const float* y = a.grad + nh * a.grad_nh + sp * a.grad_seg;
    double s = 0.0;
    if (a.cells % 4 == 0) {   // states 16 bytes apart: eight vectors of each on their way
      const f32x4_t *x4 = reinterpret_cast<const f32x4_t*>(x), *y4 = reinterpret_cast<const f32x4_t*>(y);
      const int vecs = a.cells / 4;
      for (int i0 = tid; i0 < vecs; i0 += 2048) {
        f32x4_t u[8], v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int i = min(i0 + k * 256, vecs - 1);
          u[k] = x4[i];
          v[k] = y4[i];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (i0 + k * 256 < vecs) s += (double)(fmaf(u[k][0], v[k][0], u[k][1] * v[k][1]) + fmaf(u[k][2], v[k][2], u[k][3] * v[k][3]));
      }
    } else {
      for (int i = tid; i < a.cells; i += 256) s += (double)x[i] * y[i];
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    carry = (part[0] + part[1]) + (part[2] + part[3]);
    if (e < len) carry *= (double)exp2_parts(log2_decay(load_elem(a.gate, g0 + e * a.gs.t, a.gate_f32), a.form));
    __syncthreads();
  }
  // Nothing comes from before the first token if the state there is zero: its gradient is
  // zero, and the sum's rounding errors are not.
  int starts = 1;
  if (sp == 0) {
    const float* x = a.state + nh * a.state_nh;
    starts = 0;
    if (a.cells % 4 == 0) {
      const f32x4_t* x4 = reinterpret_cast<const f32x4_t*>(x);
      const int vecs = a.cells / 4;
      for (int i0 = tid; i0 < vecs; i0 += 4096) {
        f32x4_t u[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) u[k] = x4[min(i0 + k * 256, vecs - 1)];
#pragma unroll
        for (int k = 0; k < 16; ++k) starts |= u[k][0] != 0.0f || u[k][1] != 0.0f || u[k][2] != 0.0f || u[k][3] != 0.0f;
      }
    } else {
      for (int i = tid; i < a.cells; i += 256) starts |= x[i] != 0.0f;
    }
    starts = __syncthreads_or(starts);
  }
  // 256 tokens at a time, from the end
  for (int top = e; top > b; top -= 256) {
    const int t = top - 1 - tid;
    const bool here = t >= b, live = here && t < len;
    double s = 0.0;
    if (live) s = (double)a.dq[(long)nh * a.T + t] - (double)a.dk[(long)nh * a.T + t];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double o = __shfl_up(s, d);
      if (lane >= d) s += o;
    }
    if (lane == 63) part[wave] = s;
    __syncthreads();
    double before = carry, sum = 0.0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (u < wave) before += part[u];
      sum += part[u];
    }
    carry += sum;
    if (here) {
      float r = 0.0f;
      if (live) {
        const float g = load_elem(a.gate, g0 + t * a.gs.t, a.gate_f32);
        r = (float)(before + s);
        if (a.form == kGateLogit) {
          const float x = expf(-fabsf(g));
          r *= (g >= 0.0f ? x : 1.0f) / (1.0f + x);
        }
        // nothing passes a decay of zero (the sum has rounding errors there)
        if (__builtin_amdgcn_exp2f((float)log2_decay(g, a.form)) == 0.0f) r = 0.0f;
        if (t == 0 && !starts) r = 0.0f;
      }
      const long at = n * a.os.n + t * a.os.t + h * a.os.h;
      if (a.gate_f32) reinterpret_cast<float*>(a.out)[at] = r;
      else reinterpret_cast<__bf16*>(a.out)[at] = (__bf16)r;
    }
    __syncthreads();
  }
}

// Gradients of heads that several heads read: the sum over them, in order.
// part [N * T][H][D] fp32 -> out.  3 x 1531 tokens, 6 heads of 40 and three to one: 5 us,
// a launch.
__global__ __launch_bounds__(256) void k_sum_heads(const float* part, char* out, Str os, int f32, int T, int H, int D,
                                                   int share, long count) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < count; i += (long)gridDim.x * 256) {
    const int d = (int)(i % D), hx = (int)(i / D % (H / share));
    const long nt = i / D / (H / share);
    const float* p = part + (nt * H + (long)hx * share) * D + d;
    float s = 0.0f;
    for (int u = 0; u < share; ++u) s += p[(long)u * D];
    const long at = nt / T * os.n + nt % T * os.t + hx * os.h + d;
    if (f32) reinterpret_cast<float*>(out)[at] = s;
    else reinterpret_cast<__bf16*>(out)[at] = (__bf16)s;
  }
}

// One token: state' = a state + k v^T, y = scale state'^T q.  A block has V * 2^lc
// columns of one state; its threads share the rows, kStepRows of each on their way.
// Bound by the state's bytes, in and out: 128 sequences of 16 heads of 128 x 128, 268 MB
// in 55 us (4.9 TB/s); four sequences 5 us, and 9 us with the call.
struct Step {
  const char *q, *k, *v, *gate;
  Str qs, ks, vs, gs;      // t unused
  int qd, kd, vd, gate_f32, form;
  const float* state;
  float* state_out;
  const int* slots;
  char* y;
  int N, H, K, V, S, lc, slices;
  float scale;
};

constexpr int kStepRows = 8;

template <int DT, int V>
__global__ __launch_bounds__(256) void k_step(Step a) {
  __shared__ float sum[4][64 * V];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slice = blockIdx.x % a.slices, nh = blockIdx.x / a.slices, n = nh / a.H, h = nh % a.H;
  const int lanes = 1 << a.lc, rows = 256 >> a.lc, row = tid >> a.lc, cl = (tid & (lanes - 1)) * V;
  const int c0 = slice * lanes * V, col = c0 + cl;
  const bool on = col < a.V;   // V divides a.V
  const int slot = a.slots ? a.slots[n] : n;
  const bool live = slot >= 0 && slot < a.S;
  float acc[V] = {};
  if (live && on) {
    const float dec = exp2_parts(log2_decay(load_elem(a.gate, n * a.gs.n + h * a.gs.h, a.gate_f32), a.form));
    const long base = ((long)slot * a.H + h) * a.K * a.V + col;
    const long qb = n * a.qs.n + (h / a.qd) * a.qs.h, kb = n * a.ks.n + (h / a.kd) * a.ks.h;
    const long vb = n * a.vs.n + (h / a.vd) * a.vs.h + col;
    float vv[V];
#pragma unroll
    for (int u = 0; u < V; ++u) vv[u] = load_elem(a.v, vb + u, DT == kF32);
    for (int k0 = row; k0 < a.K; k0 += rows * kStepRows) {
      Raw<V> s[kStepRows];
      float q[kStepRows], k[kStepRows];
#pragma unroll
      for (int i = 0; i < kStepRows; ++i) {
        const int kk = min(k0 + i * rows, a.K - 1);
        s[i] = *reinterpret_cast<const Raw<V>*>(a.state + base + (long)kk * a.V);
        q[i] = load_elem(a.q, qb + kk, DT == kF32);
        k[i] = load_elem(a.k, kb + kk, DT == kF32);
      }
#pragma unroll
      for (int i = 0; i < kStepRows; ++i) {
        const int kk = k0 + i * rows;
        if (kk < a.K) {
#pragma unroll
          for (int u = 0; u < V; ++u) {
            const float x = fmaf(dec, __uint_as_float(s[i][u]), k[i] * vv[u]);
            s[i][u] = __float_as_uint(x);
            acc[u] = fmaf(q[i], x, acc[u]);
          }
          *reinterpret_cast<Raw<V>*>(a.state_out + base + (long)kk * a.V) = s[i];
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < V; ++u) {
    for (int d = lanes; d < 64; d *= 2) acc[u] += __shfl_xor(acc[u], d);
    if (lane < lanes) sum[wave][cl + u] = acc[u];
  }
  __syncthreads();
  if (tid < lanes * V && c0 + tid < a.V) {
    const float y = ((sum[0][tid] + sum[1][tid]) + (sum[2][tid] + sum[3][tid])) * a.scale;
    const long at = (long)nh * a.V + c0 + tid;
    if constexpr (DT == kF32) reinterpret_cast<float*>(a.y)[at] = y;
    else reinterpret_cast<__bf16*>(a.y)[at] = (__bf16)y;
  }
}

hipError_t launch_walk(const Walk& w, const Walk* beside, int dt, hipStream_t s) {
  return dt == kBF16 ? launch_walk_bf16(w, beside, s) : launch_walk_f32(w, beside, s);
}

inline Str str(const bc_strides& s) { return {(long)s.batch, (long)s.row, (long)s.head}; }
inline size_t up(size_t v) { return (v + 255) & ~(size_t)255; }
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

// How a call is divided: segments of whole chunks, a block each.  Joining them costs a
// pass over keys and values and one over states, so a sequence stays whole up to 256
// tokens (512 where it would have three segments at most) and where each CU has one as
// it is; else two blocks a CU where segments keep 256 tokens (more would be a second
// round), or one where they keep 64.  With kept states a segment has 2048 tokens at
// most: the gates' gradients are sums over it.
// In training, bf16, rows of 128: 64 heads of 4096 tokens 436 us (8 segments), as 4 475, as
// 16 521; 384 heads of 1024 522 us, as two segments 903; 128 heads of 400 137 us, as two
// 152; 3 heads of 432 59 us (7 segments), as 4 75, whole 137.  Rows of 64, 16 heads of
// 4096 87 us (256 tokens), of 128 tokens 93.
struct Plan { int seg, segs; };
Plan plan_of(const bc_attention& a, bool keeps) {
  const long nh = (long)a.N * a.H, T = a.T;
  long segs = 1;
  if (nh < 256 && T > (nh > 64 ? 512 : 256)) segs = std::max(std::min(512 / nh, T / 256), std::min(256 / nh, ceil_div(T, 64)));
  if (keeps) segs = std::max(segs, ceil_div(T, 2048));
  const long seg = ceil_div(ceil_div(T, segs), kChunk) * kChunk;
  return {(int)seg, (int)ceil_div(T, seg)};
}

// Workspaces.  What joins the segments: their decays and the states at their
// borders; backward, what the gates' gradients are made from, and shared heads'.
struct Ws { size_t decay, entries, dots, part, part_v, total; };
Ws ws_of(const bc_attention& a, const Plan& p, bool bwd) {
  const size_t nh = (size_t)a.N * a.H;
  Ws w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up(bytes);
    return here;
  };
  if (p.segs > 1) {
    w.decay = take(nh * p.segs * sizeof(Power));
    w.entries = take(nh * (p.segs + 1) * a.Dk * a.Dv * 4);
  }
  if (bwd) {
    w.dots = take(up(nh * a.T * 4) * 2);
    // gradients by reading head: q's, then k's; and v's
    if (a.Hq < a.H || a.Hk < a.H) w.part = take(nh * a.T * a.Dk * 4);
    if (a.Hv < a.H) w.part_v = take(nh * a.T * a.Dv * 4);
  }
  w.total = at;
  return w;
}

Walk walk_of(const Attention& f) {
  Walk w{};
  const bc_attention& a = *f.a;
  w.gate = static_cast<const char*>(f.gate);
  w.gs = str(f.gs);
  w.gate_f32 = a.gate_dt == kF32;
  w.form = a.form;
  w.lengths = f.lengths;
  w.N = a.N;
  w.T = a.T;
  w.H = a.H;
  w.scale = w.kv = 1.0f;
  return w;
}

// A single token's rows may have any stride.
inline Str rows_str(const bc_strides& s, int T, int len) { return {(long)s.batch, T > 1 ? (long)s.row : len, (long)s.head}; }

struct Operand { const void* p; bc_strides s; int div, len; };
void set(Walk& w, const Operand& q, const Operand& k, const Operand& v) {
  w.q = static_cast<const char*>(q.p);
  w.k = static_cast<const char*>(k.p);
  w.v = static_cast<const char*>(v.p);
  w.qs = rows_str(q.s, w.T, q.len);
  w.ks = rows_str(k.s, w.T, k.len);
  w.vs = rows_str(v.s, w.T, v.len);
  w.qd = q.div;
  w.kd = k.div;
  w.vd = v.div;
  w.K = k.len;
  w.V = v.len;
}

}  // namespace

}  // namespace linattn

using namespace linattn;


#define BC_TRY(call)                      \
  do {                                    \
    const hipError_t e_ = (call);         \
    if (e_ != hipSuccess) return e_;      \
  } while (0)

size_t linear_attention_states_bytes(int N, int T, int H, int Dk, int Dv) {
  bc_attention a{};
  a.N = N;
  a.T = T;
  a.H = H;
  a.dt = kF32;
  return (size_t)N * H * (plan_of(a, true).segs + 1) * Dk * Dv * 4;
}

size_t linear_attention_workspace_bytes(bool bwd, const bc_attention& a) {
  const size_t keeps = ws_of(a, plan_of(a, true), bwd).total;
  return bwd ? keeps : std::max(keeps, ws_of(a, plan_of(a, false), false).total);
}

hipError_t launch_linear_attention_fwd(const Attention& f, hipStream_t s) {
  const bc_attention& a = *f.a;
  const Plan p = plan_of(a, f.states != nullptr);
  const Ws ws = ws_of(a, p, false);
  const long cells = (long)a.Dk * a.Dv, nh = (long)a.N * a.H;
  char* wsp = static_cast<char*>(f.ws);
  Walk w = walk_of(f);
  set(w, {f.q, f.qs, a.H / a.Hq, a.Dk}, {f.k, f.ks, a.H / a.Hk, a.Dk}, {f.v, f.vs, a.H / a.Hv, a.Dv});
  w.seg = p.seg;
  w.segs = p.segs;
  w.rows_first = 1;
  const long border = (p.segs + 1) * cells;   // states of one sequence and head
  if (p.segs > 1) {
    // the segments' own states, each where the state at its end belongs
    float* entry = f.states ? f.states : reinterpret_cast<float*>(wsp + ws.entries);
    w.last = entry + cells;
    w.last_nh = border;
    w.last_seg = cells;
    w.decay = reinterpret_cast<Power*>(wsp + ws.decay);
    BC_TRY(launch_walk(w, nullptr, a.dt, s));
    Joint j{};
    j.entry = entry;
    j.entry_nh = border;
    j.start = f.s0;
    j.decay = w.decay;
    j.last = f.s_last;
    j.H = a.H;
    j.segs = p.segs;
    j.cells = (int)cells;
    hipLaunchKernelGGL(k_join, dim3((unsigned)(ceil_div(cells, 256) * nh)), dim3(256), 0, s, j);
    BC_TRY(hipGetLastError());
    w.init = entry;
    w.init_nh = border;
    w.init_seg = cells;
    w.last = nullptr;
    w.decay = nullptr;
  } else {
    w.init = f.s0;
    w.init_nh = cells;
    w.last = f.s_last;
    w.last_nh = cells;
    if (f.states) {
      w.first = f.states;
      w.last2 = f.states + cells;
      w.last2_nh = border;
    }
  }
  w.y = static_cast<char*>(f.y);
  w.ys = rows_str(f.ys, a.T, a.Dv);
  w.scale = a.scale;
  return launch_walk(w, nullptr, a.dt, s);
}

hipError_t launch_linear_attention_bwd(const Attention& f, hipStream_t s) {
  const bc_attention& a = *f.a;
  const Plan p = plan_of(a, true);
  const Ws ws = ws_of(a, p, true);
  const long cells = (long)a.Dk * a.Dv, nh = (long)a.N * a.H, border = (p.segs + 1) * cells;
  char* wsp = static_cast<char*>(f.ws);
  const Operand q{f.q, f.qs, a.H / a.Hq, a.Dk}, k{f.k, f.ks, a.H / a.Hk, a.Dk}, v{f.v, f.vs, a.H / a.Hv, a.Dv},
      dy{f.gy, f.gys, 1, a.Dv};
  float* dots = reinterpret_cast<float*>(wsp + ws.dots);
  float* dots_k = reinterpret_cast<float*>(wsp + ws.dots + up(nh * a.T * 4));
  Walk forward = walk_of(f);
  forward.seg = p.seg;
  forward.segs = p.segs;
  Walk back = forward;
  back.rev = 1;
  back.kv = a.scale;

  // outputs of a walk: the gradient itself, or by reading head in the workspace,
  // to be summed
  auto out = [&](Walk& w, void* g, const bc_strides& gs, const Operand& like, size_t part) {
    const int D = like.len;
    const bool shared = like.div > 1;
    w.y = static_cast<char*>(shared ? static_cast<void*>(wsp + part) : g);
    w.ys = shared ? Str{(long)a.T * a.H * D, (long)a.H * D, D} : rows_str(gs, a.T, D);
    w.y_f32 = shared;
  };
  auto sum_heads = [&](void* g, const bc_strides& gs, const Operand& like, size_t part) -> hipError_t {
    if (like.div == 1) return hipSuccess;
    const long count = (long)a.N * a.T * (a.H / like.div) * like.len;
    hipLaunchKernelGGL(k_sum_heads, dim3((unsigned)std::min(ceil_div(count, 256), 1L << 16)), dim3(256), 0, s,
                       reinterpret_cast<const float*>(wsp + part), static_cast<char*>(g), str(gs), a.dt == kF32, a.T, a.H,
                       like.len, like.div, count);
    return hipGetLastError();
  };
  auto with_dots = [&](Walk& w, const Operand& x, float* to) {
    if (!f.ggate) return;
    w.x = static_cast<const char*>(x.p);
    w.xs = rows_str(x.s, a.T, x.len);
    w.xd = x.div;
    w.dots = to;
  };

  // Two walks at a time where one leaves CUs without a second block: 18 heads of 1531
  // tokens, 216 segments, 117 us, one by one 124; 384 segments 522 us, 540.  Where each
  // fills the card they only stand in one another's way: 512 segments 437 us one by
  // one, 471 in twos.
  const bool pairs = nh * p.segs < 512;
  Walk dq = forward;
  set(dq, dy, v, k);
  dq.init = f.states;
  dq.init_nh = border;
  dq.init_seg = cells;
  dq.scale = a.scale;
  with_dots(dq, q, dots);
  out(dq, f.gq, f.gqs, q, ws.part);

  // beside it R at the segments' ends, as far as the segments make it themselves
  back.init = f.gs_last;
  back.init_nh = cells;
  if (p.segs > 1) {
    float* entry = reinterpret_cast<float*>(wsp + ws.entries);
    Walk w = back;
    set(w, dy, q, dy);
    w.init = nullptr;
    w.rows_first = 1;
    w.last = entry;
    w.last_nh = border;
    w.last_seg = cells;
    w.decay = reinterpret_cast<Power*>(wsp + ws.decay);
    if (pairs) {
      BC_TRY(launch_walk(dq, &w, a.dt, s));
    } else {
      BC_TRY(launch_walk(dq, nullptr, a.dt, s));
      BC_TRY(launch_walk(w, nullptr, a.dt, s));
    }
    Joint j{};
    j.entry = entry;
    j.entry_nh = border;
    j.start = f.gs_last;
    j.decay = w.decay;
    j.last = f.gs0;
    j.gate = w.gate;
    j.gs = w.gs;
    j.gate_f32 = w.gate_f32;
    j.form = w.form;
    j.lengths = f.lengths;
    j.H = a.H;
    j.segs = p.segs;
    j.cells = (int)cells;
    j.rev = 1;
    hipLaunchKernelGGL(k_join, dim3((unsigned)(ceil_div(cells, 256) * nh)), dim3(256), 0, s, j);
    BC_TRY(hipGetLastError());
    back.init = entry + cells;
    back.init_nh = border;
    back.init_seg = cells;
  } else {
    BC_TRY(launch_walk(dq, nullptr, a.dt, s));
  }
  BC_TRY(sum_heads(f.gq, f.gqs, q, ws.part));

  Walk dk = back;
  set(dk, v, dy, q);
  with_dots(dk, k, dots_k);
  out(dk, f.gk, f.gks, k, ws.part);
  Walk dv = back;
  set(dv, k, q, dy);
  dv.rows_first = 1;
  out(dv, f.gv, f.gvs, v, ws.part_v);
  // grad_s0, unless k_join had it.  It may be grad_s_last, which the others read:
  // then this walk is the last.
  const bool by_dv = p.segs == 1 && f.gs0, alone = by_dv && f.gs0 == f.gs_last;
  if (by_dv) {
    dv.last = f.gs0;
    dv.last_nh = cells;
    dv.last_a0 = 1;
  }
  BC_TRY(launch_walk(dk, alone || !pairs ? nullptr : &dv, a.dt, s));
  BC_TRY(sum_heads(f.gk, f.gks, k, ws.part));

  if (f.ggate) {
    GateGrad d{};
    d.dq = dots;
    d.dk = dots_k;
    d.state = f.states;
    d.state_nh = border;
    d.grad = back.init;
    d.grad_nh = back.init_nh;
    d.grad_seg = back.init_seg;
    d.gate = back.gate;
    d.gs = back.gs;
    d.gate_f32 = back.gate_f32;
    d.form = back.form;
    d.out = static_cast<char*>(f.ggate);
    d.os = str(f.ggs);
    d.lengths = f.lengths;
    d.T = a.T;
    d.H = a.H;
    d.seg = p.seg;
    d.segs = p.segs;
    d.cells = (int)cells;
    hipLaunchKernelGGL(k_gate_grad, dim3((unsigned)(nh * p.segs)), dim3(256), 0, s, d);
    BC_TRY(hipGetLastError());
  }
  if (alone || !pairs) BC_TRY(launch_walk(dv, nullptr, a.dt, s));
  return sum_heads(f.gv, f.gvs, v, ws.part_v);
}

hipError_t launch_linear_attention_step(const Attention& f, const float* state, float* state_out, const int* slots, int S,
                                        hipStream_t s) {
  const bc_attention& a = *f.a;
  Step p{};
  p.q = static_cast<const char*>(f.q);
  p.k = static_cast<const char*>(f.k);
  p.v = static_cast<const char*>(f.v);
  p.gate = static_cast<const char*>(f.gate);
  p.qs = str(f.qs);
  p.ks = str(f.ks);
  p.vs = str(f.vs);
  p.gs = str(f.gs);
  p.qd = a.H / a.Hq;
  p.kd = a.H / a.Hk;
  p.vd = a.H / a.Hv;
  p.gate_f32 = a.gate_dt == kF32;
  p.form = a.form;
  p.state = state;
  p.state_out = state_out;
  p.slots = slots;
  p.y = static_cast<char*>(f.y);
  p.N = a.N;
  p.H = a.H;
  p.K = a.Dk;
  p.V = a.Dv;
  p.S = S;
  p.scale = a.scale;
  const int V = a.Dv % 4 == 0 ? 4 : 1;
  // whole rows of the state to a block where there are blocks enough
  p.lc = 0;
  while ((V << p.lc) < a.Dv && p.lc < 6) ++p.lc;
  auto blocks = [&]() { return (long)a.N * a.H * ceil_div(a.Dv, (long)V << p.lc); };
  while (p.lc > 2 && blocks() < 512) --p.lc;
  p.slices = (int)ceil_div(a.Dv, (long)V << p.lc);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks()), dim3(256), 0, s, p);
    return hipGetLastError();
  };
  if (a.dt == kBF16) return V == 4 ? go(k_step<kBF16, 4>) : go(k_step<kBF16, 1>);
  return V == 4 ? go(k_step<kF32, 4>) : go(k_step<kF32, 1>);
}

#undef BC_TRY

}  // namespace bc
