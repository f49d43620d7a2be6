// Linear attention with a decay for each head: how a call is divided, the joints
// between segments, the gates' gradients, and the step for single tokens.  The
// walk over segments is bc_linattn_walk.hpp's.
#include <algorithm>

#include "bc_internal.hpp"
#include "bc_linattn.hpp"

namespace bc {
namespace linattn {
namespace {

// States at the segments' borders from the segments' own: with one entry a
// border, forward (entry idx(s) holds what segment s leaves by itself) from the
// first on, backward in time from the last.  entries -> states, in place.
struct Joint {
  float* entry;
  long entry_nh;           // elements between (sequence, head)s
  const float* start;      // [nh][cells], or null: zero
  const float* decay;      // [nh][segs]
  float* last;             // [nh][cells], or null
  const char* gate;        // rev: last is times the first token's decay
  Str gs;
  int gate_f32, form;
  const int* lengths;
  int H, segs, step, border, cells, rev;   // forward: entry min((s + 1) step, border) ends segment s
};

constexpr int kJointAhead = 8;   // segments whose entries are on their way

__global__ __launch_bounds__(256) void k_join(Joint j) {
  const int blocks = (j.cells + 255) / 256, nh = blockIdx.x / blocks, cell = blockIdx.x % blocks * 256 + threadIdx.x;
  if (cell >= j.cells) return;
  float* p = j.entry + nh * j.entry_nh + cell;
  const float* dec = j.decay + (long)nh * j.segs;
  float s = j.start ? j.start[(long)nh * j.cells + cell] : 0.0f;
  p[j.rev ? (long)j.border * j.cells : 0] = s;
  auto at = [&](int i) { return (long)(j.rev ? j.segs - 1 - i : min((i + 1) * j.step, j.border)) * j.cells; };
  for (int i0 = 0; i0 < j.segs; i0 += kJointAhead) {
    float add[kJointAhead], d[kJointAhead];
#pragma unroll
    for (int u = 0; u < kJointAhead; ++u) {
      const int i = min(i0 + u, j.segs - 1);
      add[u] = p[at(i)];
      d[u] = dec[j.rev ? j.segs - 1 - i : i];
    }
#pragma unroll
    for (int u = 0; u < kJointAhead; ++u) {
      if (i0 + u < j.segs) {
        s = fmaf(d[u], s, add[u]);
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

// The gates' gradients of one span: the sum of q . dq - k . dk from a token to
// the span's end, and what crosses that end, <state, gradient> of the border.
struct GateGrad {
  const float *dq, *dk;          // [nh][T]: q_t . dq_t, k_t . dk_t
  const float* state;            // the state after the span: entry nh * state_nh + (span + 1) cells
  long state_nh;
  const float* grad;             // its gradient, before the next token's decay; null: zero
  long grad_nh, grad_span;
  const char* gate;
  Str gs;
  int gate_f32, form;
  char* out;
  Str os;
  const int* lengths;
  int T, H, span, spans, cells;
};

__global__ __launch_bounds__(256) void k_gate_grad(GateGrad a) {
  __shared__ double part[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sp = blockIdx.x % a.spans, nh = blockIdx.x / a.spans, n = nh / a.H, h = nh % a.H;
  const int len = a.lengths ? min(max(a.lengths[n], 0), a.T) : a.T;
  const int b = sp * a.span, e = min(b + a.span, a.T);
  const long g0 = n * a.gs.n + h * a.gs.h;
  double carry = 0.0;
  if (a.grad && b < len) {
    const float* x = a.state + nh * a.state_nh + (long)(sp + 1) * a.cells;
    const float* y = a.grad + nh * a.grad_nh + sp * a.grad_span;
    double s = 0.0;
    int i = tid * 4;
    for (; i + 3 < a.cells; i += 1024) {
      float t = 0.0f;
#pragma unroll
      for (int u = 0; u < 4; ++u) t = fmaf(x[i + u], y[i + u], t);
      s += t;
    }
    for (; i < a.cells; ++i) s += (double)x[i] * y[i];
#pragma unroll
    for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    carry = (part[0] + part[1]) + (part[2] + part[3]);
    if (e < len) carry *= (double)exp2_parts(log2_decay(load_elem(a.gate, g0 + e * a.gs.t, a.gate_f32), a.form));
    __syncthreads();
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
      }
      const long at = n * a.os.n + t * a.os.t + h * a.os.h;
      if (a.gate_f32) reinterpret_cast<float*>(a.out)[at] = r;
      else reinterpret_cast<__bf16*>(a.out)[at] = (__bf16)r;
    }
    __syncthreads();
  }
}

// Gradients of heads that several heads read: the sum over them, in order.
// part [N * T][H][D] fp32 -> out.
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
// columns of one state; its threads share the rows, kRows of each on their way.
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

hipError_t launch_walk(const Walk& w, int dt, hipStream_t s) {
  return dt == kBF16 ? launch_walk_bf16(w, s) : launch_walk_f32(w, s);
}

inline Str str(const bc_strides& s) { return {(long)s.batch, (long)s.row, (long)s.head}; }
inline size_t up(size_t v) { return (v + 255) & ~(size_t)255; }
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

// How a call is divided.  Spans: the backward's segments, between kept states;
// as long as two blocks on each of 256 CUs allow, 128 to 1024 tokens (the gates'
// gradients sum over a span).  The forward's segments are whole spans.
struct Plan { int span, spans, seg, segs; };
Plan plan_of(int N, int T, int H) {
  const long nh = (long)N * H;
  Plan p;
  p.span = (int)std::min(1024L, std::max(128L, nh * T / 512 / 64 * 64));
  p.spans = (int)ceil_div(T, p.span);
  const long want = std::min<long>(p.spans, std::max(1L, 512 / nh));
  const int per = (int)ceil_div(p.spans, want);
  p.seg = per * p.span;
  p.segs = (int)ceil_div(p.spans, per);
  return p;
}

struct FwdWs { size_t decay, entries, total; };
FwdWs fwd_ws(const bc_attention& a, const Plan& p) {
  FwdWs w{};
  if (p.segs == 1) return w;
  const size_t nh = (size_t)a.N * a.H;
  w.entries = up(nh * p.segs * 4);
  w.total = w.entries + up(nh * (p.segs + 1) * a.Dk * a.Dv * 4);
  return w;
}

struct BwdWs { size_t decay, entries, dots, part, total; };
BwdWs bwd_ws(const bc_attention& a, const Plan& p) {
  BwdWs w{};
  const size_t nh = (size_t)a.N * a.H;
  size_t at = 0;
  if (p.spans > 1) {
    w.entries = up(nh * p.spans * 4);
    at = w.entries + up(nh * (p.spans + 1) * a.Dk * a.Dv * 4);
  }
  w.dots = at;
  w.part = at + up(nh * a.T * 4) * 2;
  size_t d = 0;   // gradients by reading head, summed afterwards; one at a time
  if (a.Hq < a.H || a.Hk < a.H) d = a.Dk;
  if (a.Hv < a.H) d = std::max(d, (size_t)a.Dv);
  w.total = w.part + up(nh * a.T * d * 4);
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

struct Operand { const void* p; bc_strides s; int div, len; };
void set(Walk& w, const Operand& q, const Operand& k, const Operand& v) {
  w.q = static_cast<const char*>(q.p);
  w.k = static_cast<const char*>(k.p);
  w.v = static_cast<const char*>(v.p);
  w.qs = str(q.s);
  w.ks = str(k.s);
  w.vs = str(v.s);
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

long linear_attention_blocks(int N, int T, int H) { return (long)N * H * plan_of(N, T, H).spans; }

size_t linear_attention_states_bytes(int N, int T, int H, int Dk, int Dv) {
  return (size_t)N * H * (plan_of(N, T, H).spans + 1) * Dk * Dv * 4;
}

size_t linear_attention_workspace_bytes(bool bwd, const bc_attention& a) {
  const Plan p = plan_of(a.N, a.T, a.H);
  return bwd ? bwd_ws(a, p).total : fwd_ws(a, p).total;
}

hipError_t launch_linear_attention_fwd(const Attention& f, hipStream_t s) {
  const bc_attention& a = *f.a;
  const Plan p = plan_of(a.N, a.T, a.H);
  const FwdWs ws = fwd_ws(a, p);
  const long cells = (long)a.Dk * a.Dv;
  char* wsp = static_cast<char*>(f.ws);
  Walk w = walk_of(f);
  set(w, {f.q, f.qs, a.H / a.Hq, a.Dk}, {f.k, f.ks, a.H / a.Hk, a.Dk}, {f.v, f.vs, a.H / a.Hv, a.Dv});
  w.seg = p.seg;
  w.segs = p.segs;
  w.sk = a.Dv;
  w.sv = 1;
  w.span = p.span;
  if (p.segs > 1) {
    const int per = p.seg / p.span;
    Joint j{};
    j.entry = f.states ? f.states : reinterpret_cast<float*>(wsp + ws.entries);
    j.step = f.states ? per : 1;
    j.border = f.states ? p.spans : p.segs;
    j.entry_nh = (j.border + 1) * cells;
    // the segments' own states and decays, in the entries of their ends.  The
    // last one's entry is the border's.
    w.last = j.entry + j.step * cells;
    w.last_nh = j.entry_nh;
    w.last_seg = j.step * cells;
    w.last_max = (j.border - j.step) * cells;
    w.decay = reinterpret_cast<float*>(wsp + ws.decay);
    BC_TRY(launch_walk(w, a.dt, s));
    j.start = f.s0;
    j.decay = w.decay;
    j.last = f.s_last;
    j.H = a.H;
    j.segs = p.segs;
    j.cells = (int)cells;
    hipLaunchKernelGGL(k_join, dim3((unsigned)(ceil_div(cells, 256) * a.N * a.H)), dim3(256), 0, s, j);
    BC_TRY(hipGetLastError());
    w.init = j.entry;
    w.init_nh = j.entry_nh;
    w.init_seg = j.step * cells;
    w.last = nullptr;
    w.decay = nullptr;
  } else {
    w.init = f.s0;
    w.init_nh = cells;
    w.last = f.s_last;
    w.last_nh = cells;
    if (f.states) {
      w.last2 = f.states + p.spans * cells;
      w.last2_nh = (p.spans + 1) * cells;
    }
  }
  if (f.states) {
    w.save = f.states;
    w.save_nh = (p.spans + 1) * cells;
  }
  w.y = static_cast<char*>(f.y);
  w.ys = str(f.ys);
  w.scale = a.scale;
  return launch_walk(w, a.dt, s);
}

hipError_t launch_linear_attention_bwd(const Attention& f, hipStream_t s) {
  const bc_attention& a = *f.a;
  const Plan p = plan_of(a.N, a.T, a.H);
  const BwdWs ws = bwd_ws(a, p);
  const long cells = (long)a.Dk * a.Dv, nh = (long)a.N * a.H;
  char* wsp = static_cast<char*>(f.ws);
  const Operand q{f.q, f.qs, a.H / a.Hq, a.Dk}, k{f.k, f.ks, a.H / a.Hk, a.Dk}, v{f.v, f.vs, a.H / a.Hv, a.Dv},
      dy{f.gy, f.gys, 1, a.Dv};
  float* dots = f.ggate ? reinterpret_cast<float*>(wsp + ws.dots) : nullptr;
  float* dots_k = f.ggate ? reinterpret_cast<float*>(wsp + ws.dots + up(nh * a.T * 4)) : nullptr;
  Walk base = walk_of(f);
  base.seg = p.span;
  base.segs = p.spans;
  base.span = p.span;

  // R at the spans' ends
  const float* grad = f.gs_last;
  long grad_nh = cells, grad_span = 0;
  if (p.spans > 1) {
    float* entry = reinterpret_cast<float*>(wsp + ws.entries);
    Walk w = base;
    set(w, dy, q, dy);
    w.rev = 1;
    w.sk = a.Dv;
    w.sv = 1;
    w.kv = a.scale;
    w.last = entry;
    w.last_nh = (p.spans + 1) * cells;
    w.last_seg = cells;
    w.last_max = p.spans * cells;
    w.decay = reinterpret_cast<float*>(wsp + ws.decay);
    BC_TRY(launch_walk(w, a.dt, s));
    Joint j{};
    j.entry = entry;
    j.entry_nh = (p.spans + 1) * cells;
    j.start = f.gs_last;
    j.decay = w.decay;
    j.last = f.gs0;
    j.gate = base.gate;
    j.gs = base.gs;
    j.gate_f32 = base.gate_f32;
    j.form = base.form;
    j.lengths = f.lengths;
    j.H = a.H;
    j.segs = p.spans;
    j.border = p.spans;
    j.cells = (int)cells;
    j.rev = 1;
    hipLaunchKernelGGL(k_join, dim3((unsigned)(ceil_div(cells, 256) * nh)), dim3(256), 0, s, j);
    BC_TRY(hipGetLastError());
    grad = entry + cells;
    grad_nh = j.entry_nh;
    grad_span = cells;
  }

  auto out = [&](Walk& w, void* g, const bc_strides& gs, int share, int D) -> hipError_t {
    w.y = static_cast<char*>(share > 1 ? static_cast<void*>(wsp + ws.part) : g);
    w.ys = share > 1 ? Str{(long)a.T * a.H * D, (long)a.H * D, D} : str(gs);
    w.y_f32 = share > 1 || a.dt == kF32;
    BC_TRY(launch_walk(w, a.dt, s));
    if (share == 1) return hipSuccess;
    const long count = (long)a.N * a.T * (a.H / share) * D;
    hipLaunchKernelGGL(k_sum_heads, dim3((unsigned)std::min(ceil_div(count, 256), 1L << 16)), dim3(256), 0, s,
                       reinterpret_cast<const float*>(wsp + ws.part), static_cast<char*>(g), str(gs), a.dt == kF32, a.T, a.H,
                       D, share, count);
    return hipGetLastError();
  };

  Walk w = base;   // dq
  set(w, dy, v, k);
  w.init = f.states;
  w.init_nh = (p.spans + 1) * cells;
  w.init_seg = cells;
  w.sk = 1;
  w.sv = a.Dv;
  w.scale = a.scale;
  if (dots) {
    w.x = static_cast<const char*>(q.p);
    w.xs = str(q.s);
    w.xd = q.div;
    w.dots = dots;
  }
  BC_TRY(out(w, f.gq, f.gqs, q.div, a.Dk));

  w = base;   // dk
  set(w, v, dy, q);
  w.rev = 1;
  w.kv = a.scale;
  w.init = grad;
  w.init_nh = grad_nh;
  w.init_seg = grad_span;
  w.sk = 1;
  w.sv = a.Dv;
  if (dots) {
    w.x = static_cast<const char*>(k.p);
    w.xs = str(k.s);
    w.xd = k.div;
    w.dots = dots_k;
  }
  BC_TRY(out(w, f.gk, f.gks, k.div, a.Dk));

  if (f.ggate) {
    GateGrad d{};
    d.dq = dots;
    d.dk = dots_k;
    d.state = f.states;
    d.state_nh = (p.spans + 1) * cells;
    d.grad = grad;
    d.grad_nh = grad_nh;
    d.grad_span = grad_span;
    d.gate = base.gate;
    d.gs = base.gs;
    d.gate_f32 = base.gate_f32;
    d.form = base.form;
    d.out = static_cast<char*>(f.ggate);
    d.os = str(f.ggs);
    d.lengths = f.lengths;
    d.T = a.T;
    d.H = a.H;
    d.span = p.span;
    d.spans = p.spans;
    d.cells = (int)cells;
    hipLaunchKernelGGL(k_gate_grad, dim3((unsigned)(nh * p.spans)), dim3(256), 0, s, d);
    BC_TRY(hipGetLastError());
  }

  w = base;   // dv, last: grad_s0 may be grad_s_last, which the others read
  set(w, k, q, dy);
  w.rev = 1;
  w.kv = a.scale;
  w.init = grad;
  w.init_nh = grad_nh;
  w.init_seg = grad_span;
  w.sk = a.Dv;
  w.sv = 1;
  if (p.spans == 1) {
    w.last = f.gs0;
    w.last_nh = cells;
    w.last_a0 = 1;
  }
  return out(w, f.gv, f.gvs, v.div, a.Dv);
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
