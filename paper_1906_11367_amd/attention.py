"""A linear-attention block: norm, projections, attention with a decay for each
head, gated norm of the heads, projection, norm, residual sum.

  p = norm(x) w_pre  @ w_in          q | k | v | output gate | decay logits
  o = linear attention of q, k, v with a = sigmoid(decay logit), scale Dk^-1/2
  m = norm(o) w_head by head * silu(output gate)
  r = x + res_scale * norm(m @ w_out) w_post

It stands where the recurrent layer does (recurrent.py), with a matrix for each
head's state in place of one number for each channel.  LinearAttentionPlan trains
it on tokens [N, T, C] in fp32 or bf16; LinearAttentionServer runs trained weights
in 8-bit codes: prompts, then one token at a time for sequences whose states live
in a pool.  Every arithmetic step runs in libboxconv's kernels; torch holds the
memory.
"""
from __future__ import annotations

import dataclasses

import torch

from . import boxconv as bc


def _columns(H, Hk, Dk, Dv):
    """Where q, k, v, the output gate and the decay logits stand in the
    projection's rows, and the rows' length (each part starts on 16 bytes)."""
    up = lambda n: (n + 7) // 8 * 8
    at, out = 0, []
    for n in (H * Dk, Hk * Dk, Hk * Dv, H * Dv, H):
        out.append((at, n))
        at += up(n)
    return out, at


class _Shape:
    """Views of the projection's parts, and sizes that both uses share."""

    def __init__(self, H, Hk, Dk, Dv):
        self.H, self.Hk, self.Dk, self.Dv = H, Hk, Dk, Dv
        self.columns, self.width = _columns(H, Hk, Dk, Dv)
        self.scale = Dk ** -0.5

    def parts(self, p):
        """p [..., width] -> q [..., H, Dk], k, v [..., Hk, D], gate [..., H * Dv], logits [..., H]."""
        cut = [p[..., at:at + n] for at, n in self.columns]
        heads = ((self.H, self.Dk), (self.Hk, self.Dk), (self.Hk, self.Dv))
        return [c.unflatten(-1, h) for c, h in zip(cut, heads)] + cut[3:]


@dataclasses.dataclass
class LinearAttentionPlan:
    N: int
    T: int                 # tokens of a sequence
    C: int                 # channels of x
    H: int                 # heads
    Dk: int
    Dv: int
    Hk: int | None = None  # heads of keys and values (None: H), a divisor of H
    dtype: str = "f32"     # 'f32' | 'bf16': activations, and the products' operands
    eps: float = 1e-6
    with_backward: bool = True
    device: str = "cuda"

    def __post_init__(self):
        if self.dtype not in ("f32", "bf16"):
            raise ValueError("dtype must be 'f32' or 'bf16'")
        N, T, C, H = self.N, self.T, self.C, self.H
        self.Hk = self.Hk or H
        if H % self.Hk:
            raise ValueError("Hk must divide H")
        if N * T > 65536:
            raise ValueError("N * T must not exceed 65536 (the products' rows)")
        self.shape = _Shape(H, self.Hk, self.Dk, self.Dv)
        self.bf16 = self.dtype == "bf16"
        self.compute = bc.BC_BF16 if self.bf16 else bc.BC_F32
        self.t = torch.bfloat16 if self.bf16 else torch.float32
        W, E = self.shape.width, H * self.Dv
        dev = torch.device(self.device)
        act = lambda *s: torch.empty(s, dtype=self.t, device=dev)
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=dev)
        self.xn, self.p, self.o, self.m = act(N, T, C), act(N, T, W), act(N, T, H, self.Dv), act(N, T, E)
        self.z, self.r = act(N, T, C), act(N, T, C)
        self.s_last = f32(N, H, self.Dk, self.Dv)
        code = bc.BC_BF16 if self.bf16 else bc.BC_F32
        sizes = (N, T, H, H, self.Hk, self.Hk, self.Dk, self.Dv, code)
        ws = [bc.linear_attention_workspace_bytes(0, *sizes)]
        # a product in fp32 that a cast follows
        self.wide = f32(N * T * max(W, C, E)) if self.bf16 else None
        self.states = None
        if self.with_backward:
            self.states = bc.linear_attention_states(N, T, H, self.Dk, self.Dv, dev)
            # (columns between the parts have no gradient)
            self.dp = torch.zeros((N, T, W), dtype=self.t, device=dev)
            self.dz, self.dm, self.do = act(N, T, C), act(N, T, E), act(N, T, H, self.Dv)
            self.dr, self.dxn, self.dx = act(N, T, C), act(N, T, C), act(N, T, C)
            self.ds0 = f32(N, H, self.Dk, self.Dv)
            self.grads = {"w_pre": f32(C), "w_in": f32(C, W), "w_head": f32(E), "w_out": f32(E, C), "w_post": f32(C),
                          "res_scale": f32(C)}
            ws.append(bc.linear_attention_workspace_bytes(1, *sizes))
            ws += [bc.block_norm_workspace_bytes(N * T, c) for c in (C, E)]
            for k, p in ((C, W), (E, C)):
                ws += [bc.mix_workspace_bytes(mode, 1, N * T, k, p, self.compute)
                       for mode in (bc.BC_MIX_BWD_WEIGHT, bc.BC_MIX_BWD_DATA)]
        for k, p in ((C, W), (E, C)):
            ws.append(bc.mix_workspace_bytes(bc.BC_MIX_FWD, 1, N * T, k, p, self.compute))
        # one workspace: the calls run in order on the caller's stream
        self.ws = torch.empty(max(*ws, 16), dtype=torch.uint8, device=dev)

    # The products of rows of tokens: the mix's operands with the tokens in its
    # weights' place, [rows, K] @ [K, P] and the two that its backward has.
    def _product(self, mode, a, b, out, k, p):
        to = out
        if self.bf16 and out.dtype is not torch.float32:
            to = self.wide[:out.numel()]
        bc.pointwise_mix(mode, a, b, to, 1, self.N * self.T, k, p, self.compute, ws=self.ws)
        if to is not out:
            bc.bc_cast_bf16(to, out)
        return out

    def _matrices(self, w, what):
        # (the products see numbers of elements alone)
        E = self.H * self.Dv
        bc._need(w["w_in"], (self.C, self.shape.width), (torch.float32, torch.bfloat16), what, "w_in")
        bc._need(w["w_out"], (E, self.C), (torch.float32, torch.bfloat16), what, "w_out")

    def forward(self, x: torch.Tensor, w: dict, s0: torch.Tensor | None = None, lengths: torch.Tensor | None = None):
        """x [N, T, C] of the plan's type; w: w_pre [C], w_in [C, width], w_head
        [H * Dv], w_out [H * Dv, C], w_post [C], res_scale [C], fp32 each
        -> (r [N, T, C], s_last [N, H, Dk, Dv])."""
        s, E = self.shape, self.H * self.Dv
        bc._need(x, (self.N, self.T, self.C), self.t, "LinearAttentionPlan.forward", "x")
        self._matrices(w, "LinearAttentionPlan.forward")
        bc.block_norm_fwd(x, w_pre=w["w_pre"], y=self.xn, eps=self.eps)
        self._product(bc.BC_MIX_FWD, self.xn, w["w_in"], self.p, self.C, s.width)
        q, k, v, gate, logits = s.parts(self.p)
        bc.linear_attention_fwd(q, k, v, logits, self.o, s0=s0, s_last=self.s_last, lengths=lengths, states=self.states,
                                scale=s.scale, ws=self.ws)
        bc.block_norm_fwd(self.o.flatten(2), gate=gate, w_post=w["w_head"], r=self.m, groups=self.H, eps=self.eps)
        self._product(bc.BC_MIX_FWD, self.m, w["w_out"], self.z, E, self.C)
        bc.block_norm_fwd(self.z, x=x, w_post=w["w_post"], res_scale=w["res_scale"], r=self.r, groups=1, eps=self.eps)
        return self.r, self.s_last

    def backward(self, x: torch.Tensor, w: dict, grad_r: torch.Tensor, grad_s_last: torch.Tensor | None = None,
                 lengths: torch.Tensor | None = None):
        """After the forward of the same arguments: (dx, the weights' gradients, ds0)."""
        s, E, g = self.shape, self.H * self.Dv, self.grads
        bc._need(x, (self.N, self.T, self.C), self.t, "LinearAttentionPlan.backward", "x")
        bc._need(grad_r, (self.N, self.T, self.C), self.t, "LinearAttentionPlan.backward", "grad_r")
        self._matrices(w, "LinearAttentionPlan.backward")
        bc.block_norm_bwd(self.z, x=x, w_post=w["w_post"], res_scale=w["res_scale"], grad_r=grad_r, grad_z=self.dz,
                          grad_x=self.dr, grad_w_post=g["w_post"], grad_res_scale=g["res_scale"], groups=1, eps=self.eps,
                          ws=self.ws)
        self._product(bc.BC_MIX_BWD_DATA, self.m, self.dz, g["w_out"], E, self.C)
        self._product(bc.BC_MIX_BWD_WEIGHT, self.dz, w["w_out"], self.dm, E, self.C)
        q, k, v, gate, logits = s.parts(self.p)
        dq, dk, dv, dgate, dlogits = s.parts(self.dp)
        bc.block_norm_bwd(self.o.flatten(2), gate=gate, w_post=w["w_head"], grad_r=self.dm, grad_z=self.do.flatten(2),
                          grad_gate=dgate, grad_w_post=g["w_head"], groups=self.H, eps=self.eps, ws=self.ws)
        bc.linear_attention_bwd(q, k, v, logits, self.states, self.do, dq, dk, dv, dlogits, grad_s_last=grad_s_last,
                                grad_s0=self.ds0, lengths=lengths, scale=s.scale, ws=self.ws)
        self._product(bc.BC_MIX_BWD_DATA, self.xn, self.dp, g["w_in"], self.C, s.width)
        self._product(bc.BC_MIX_BWD_WEIGHT, self.dp, w["w_in"], self.dxn, self.C, s.width)
        bc.block_norm_bwd(x, w_pre=w["w_pre"], grad_r=self.dr, grad_y=self.dxn, grad_z=self.dx, grad_w_pre=g["w_pre"],
                          eps=self.eps, ws=self.ws)
        return self.dx, g, self.ds0


class LinearAttentionServer:
    """Inference of the block in 8-bit codes: w as LinearAttentionPlan.forward takes
    it, its two matrices turned into codes once; the states of up to `slots`
    sequences are rows of a pool, fp32, zero at first.  A slot outside the pool
    marks an idle row of a batch: it changes no state, and attention gives it
    zeros (its r is x)."""

    _rows = None

    def __init__(self, w: dict, H: int, Dk: int, Dv: int, slots: int, Hk: int | None = None,
                 dtype: torch.dtype = torch.bfloat16, eps: float = 1e-6):
        self.shape = _Shape(H, Hk or H, Dk, Dv)
        C = w["w_pre"].shape[0]
        if w["w_in"].shape != (C, self.shape.width) or w["w_out"].shape != (H * Dv, C):
            raise ValueError(f"w_in must be [{C}, {self.shape.width}] and w_out [{H * Dv}, {C}]")
        self.w, self.C, self.dtype, self.eps = w, C, dtype, eps
        self.w_in, self.w_out = self._codes(w["w_in"]), self._codes(w["w_out"])
        self.state = torch.zeros((slots, H, Dk, Dv), dtype=torch.float32, device=w["w_in"].device)

    @property
    def state(self) -> torch.Tensor:
        """The pool [slots, H, Dk, Dv]: read and written in place, or set (copied).  Setting
        as many slots leaves it where it is, so that graphs captured before work on it."""
        return self._state

    @state.setter
    def state(self, value: torch.Tensor):
        if self._rows is not None and value.shape[1:] != self._rows.shape[1:]:
            raise ValueError(f"state must be [slots, {', '.join(map(str, self._rows.shape[1:]))}]")
        if self._rows is None or value.shape[0] + 1 != self._rows.shape[0]:
            # a row more, always zero: prefill's idle rows start and end there
            self._rows = torch.zeros((value.shape[0] + 1, *value.shape[1:]), dtype=torch.float32, device=value.device)
            self._state = self._rows[:-1]
        elif value.untyped_storage().data_ptr() == self._rows.untyped_storage().data_ptr():
            value = value.clone()   # the pool's own cells, in another order
        self._state.copy_(value)

    @staticmethod
    def _codes(w):
        w = w.t().contiguous()
        q = torch.empty((w.shape[0], bc.i8_pitch(w.shape[1])), dtype=torch.int8, device=w.device)
        return bc.quantize_i8(w, q, torch.empty(w.shape[0], dtype=torch.float32, device=w.device))

    def _new(self, *shape):
        return torch.empty(shape, dtype=self.dtype, device=self._state.device)

    def _into(self, x):
        xn = self._new(*x.shape)
        bc.block_norm_fwd(x, w_pre=self.w["w_pre"], y=xn, eps=self.eps)
        return self.shape.parts(bc.pointwise_mix_i8(*self.w_in, xn, self._new(*x.shape[:-1], self.shape.width)))

    def _out_of(self, x, o, gate):
        o = o.flatten(-2)
        m, r = self._new(*o.shape), self._new(*x.shape)
        bc.block_norm_fwd(o, gate=gate, w_post=self.w["w_head"], r=m, groups=self.shape.H, eps=self.eps)
        z = bc.pointwise_mix_i8(*self.w_out, m, self._new(*x.shape))
        bc.block_norm_fwd(z, x=x, w_post=self.w["w_post"], res_scale=self.w["res_scale"], r=r, groups=1, eps=self.eps)
        return r

    def prefill(self, x: torch.Tensor, slots: torch.Tensor, lengths: torch.Tensor | None = None, fresh: bool = True):
        """Prompts x [N, T, C] of sequences slots [N] (distinct, but for idle rows)
        -> r [N, T, C]; their rows of the pool take the states at each one's length.
        fresh: from zero states, otherwise from the pool's."""
        N, T = x.shape[:2]
        bc._need(x, (N, T, self.C), self.dtype, "prefill", "x")
        bc._need(slots, (N,), (torch.int32, torch.int64), "prefill", "slots")
        bc._need(lengths, (N,), torch.int32, "prefill", "lengths")
        q, k, v, gate, logits = self._into(x)
        # an idle row is a sequence of no tokens in the pool's extra row
        S, rows = self._state.shape[0], slots.long()
        idle = (rows < 0) | (rows >= S)
        rows = rows.masked_fill(idle, S)
        if lengths is None:
            lengths = torch.full((N,), T, dtype=torch.int32, device=x.device)
        lengths = lengths.masked_fill(idle, 0)
        s = torch.empty((N, *self._rows.shape[1:]), dtype=torch.float32, device=x.device) if fresh else self._rows[rows]
        o = bc.linear_attention_fwd(q, k, v, logits, self._new(N, T, self.shape.H, self.shape.Dv),
                                    s0=None if fresh else s, s_last=s, lengths=lengths, scale=self.shape.scale)
        self._rows[rows] = s
        return self._out_of(x, o, gate)

    def step(self, x: torch.Tensor, slots: torch.Tensor | None = None):
        """One token x [N, C] of each of N sequences (slots [N] int32, or None: the
        pool's first N rows) -> r [N, C]; the pool is updated."""
        N = x.shape[0]
        bc._need(x, (N, self.C), self.dtype, "step", "x")
        q, k, v, gate, logits = self._into(x)
        o = bc.linear_attention_step(q, k, v, logits, self._state, self._new(N, self.shape.H, self.shape.Dv), slots=slots,
                                     scale=self.shape.scale)
        return self._out_of(x, o, gate)
