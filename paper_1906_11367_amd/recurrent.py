"""A recurrent layer: 1x1 mix in, gated scan along the sequence, 1x1 mix out.

The box-convolution layer filters each channel on its own and then mixes the
channels; this is the same pair along a sequence, the box filter replaced by a
gated linear recurrence:

  p = w_in x              gate = p[:D], v = p[D:]     (w_in [2D, C])
  h_t = a_t h_{t-1} + (1 - a_t) v_t,  a = sigmoid(gate)   (BC_GATE_LOGIT)
  z = w_out h                                          (w_out [M, D])

RecurrentPlan trains it on maps [N, C, T] (the pixels of a box layer's output in
raster order, or any features with time contiguous), its mixes on MFMA in fp32
or bf16.  RecurrentServer runs trained weights in 8-bit codes: prompts in either
layout, then one token at a time for sequences whose states live in a pool.
Every arithmetic step runs in libboxconv's kernels; torch holds the memory.
"""
from __future__ import annotations

import dataclasses

import torch

from . import boxconv as bc


@dataclasses.dataclass
class RecurrentPlan:
    N: int
    C: int                 # input channels
    T: int                 # steps (pixels) of a sequence
    D: int                 # states
    M: int                 # output channels
    mix_dtype: str = "f32"     # 'f32' | 'bf16': the mixes' compute type
    x_dtype: torch.dtype | None = None     # the one type of x that is taken (None: fp32, or bf16 with a bf16 mix)
    form: int = bc.BC_GATE_LOGIT
    with_backward: bool = True
    device: str = "cuda"

    def __post_init__(self):
        if self.mix_dtype not in ("f32", "bf16"):
            raise ValueError("mix_dtype must be 'f32' or 'bf16'")
        types = (torch.float32, torch.bfloat16) if self.mix_dtype == "bf16" else (torch.float32,)
        if self.x_dtype is not None and self.x_dtype not in types:
            raise ValueError("x must be fp32, or bf16 with a bf16 mix")
        self.x_types = types if self.x_dtype is None else (self.x_dtype,)
        if self.D * self.T % 8:
            raise ValueError("D * T must be a multiple of 8 (gate and input are 16-byte aligned halves)")
        dev = torch.device(self.device)
        N, C, T, D, M = self.N, self.C, self.T, self.D, self.M
        bf16 = self.mix_dtype == "bf16"
        self.compute = bc.BC_BF16 if bf16 else bc.BC_F32
        self.operand = torch.bfloat16 if bf16 else torch.float32
        f32 = dict(dtype=torch.float32, device=dev)
        self.p = torch.empty((N, 2 * D, T), **f32)
        # the scan writes the second mix's operand, the backward scan the first
        # one's gradient operand, in the mixes' type: bitwise what the mixes
        # would round themselves, read at half the bytes
        self.h = torch.empty((N, D, T), dtype=self.operand, device=dev)
        self.h_last = torch.empty((N, D), **f32)
        self.z = torch.empty((N, M, T), **f32)
        self.states = None
        ws = [bc.gated_scan_workspace_bytes(0, N, T, D, bc.BC_F32, bc.BC_MAPS)]
        if self.with_backward:
            self.states = bc.gated_scan_states(N, T, D, torch.float32, bc.BC_MAPS, dev)
            self.dh = torch.empty((N, D, T), **f32)
            self.dp = torch.empty((N, 2 * D, T), dtype=self.operand, device=dev)
            self.dx = torch.empty((N, C, T), **f32)
            self.dw_in = torch.empty((2 * D, C), **f32)
            self.dw_out = torch.empty((M, D), **f32)
            self.dh0 = torch.empty((N, D), **f32)
            ws.append(bc.gated_scan_workspace_bytes(1, N, T, D, bc.BC_F32, bc.BC_MAPS))
            for m, k in ((M, D), (2 * D, C)):
                for mode in (bc.BC_MIX_BWD_WEIGHT, bc.BC_MIX_BWD_DATA):
                    ws.append(bc.mix_workspace_bytes(mode, N, m, k, T, self.compute))
        # one workspace: the calls run in order on the caller's stream
        self.ws = torch.empty(max(*ws, 16), dtype=torch.uint8, device=dev)

    def _mix(self, mode, a, b, out, m, k):
        return bc.pointwise_mix(mode, a, b, out, self.N, m, k, self.T, self.compute, ws=self.ws)

    def forward(self, x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, h0: torch.Tensor | None = None,
                lengths: torch.Tensor | None = None):
        """x [N, C, T] -> (z [N, M, T], h_last [N, D])."""
        D = self.D
        bc._need(x, None, self.x_types, "RecurrentPlan.forward", "x")
        self._mix(bc.BC_MIX_FWD, w_in, x, self.p, 2 * D, self.C)
        bc.gated_scan_fwd(self.p[:, :D], self.p[:, D:], self.h, h0=h0, h_last=self.h_last, lengths=lengths,
                          states=self.states, form=self.form, layout=bc.BC_MAPS, ws=self.ws)
        self._mix(bc.BC_MIX_FWD, w_out, self.h, self.z, self.M, D)
        return self.z, self.h_last

    def backward(self, x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, grad_z: torch.Tensor,
                 grad_h_last: torch.Tensor | None = None, lengths: torch.Tensor | None = None):
        """After the forward of the same arguments: (dx, dw_in, dw_out, dh0)."""
        D = self.D
        bc._need(x, None, self.x_types, "RecurrentPlan.backward", "x")
        self._mix(bc.BC_MIX_BWD_WEIGHT, grad_z, self.h, self.dw_out, self.M, D)
        self._mix(bc.BC_MIX_BWD_DATA, w_out, grad_z, self.dh, self.M, D)
        bc.gated_scan_bwd(self.p[:, :D], self.p[:, D:], self.states, self.dh, self.dp[:, :D], self.dp[:, D:],
                          grad_h_last=grad_h_last, grad_h0=self.dh0, lengths=lengths, form=self.form,
                          layout=bc.BC_MAPS, ws=self.ws)
        self._mix(bc.BC_MIX_BWD_WEIGHT, self.dp, x, self.dw_in, 2 * D, self.C)
        self._mix(bc.BC_MIX_BWD_DATA, w_in, self.dp, self.dx, 2 * D, self.C)
        return self.dx, self.dw_in, self.dw_out, self.dh0


class RecurrentServer:
    """Inference of the layer in 8-bit codes.  w_in [2D, C] and w_out [M, D] (fp32
    or bf16) are turned into codes once; the states of up to `slots` sequences
    are rows of a pool, fp32, zero at first.  A slot outside the pool marks an idle
    row of a batch: it changes no state, and its z is that of a zero state (b_out)."""

    def __init__(self, w_in: torch.Tensor, w_out: torch.Tensor, slots: int, b_in: torch.Tensor | None = None,
                 b_out: torch.Tensor | None = None, form: int = bc.BC_GATE_LOGIT,
                 dtype: torch.dtype = torch.bfloat16):
        two_d, self.C = w_in.shape
        self.M, self.D = w_out.shape
        if two_d != 2 * self.D or self.D % 8:
            raise ValueError("w_in must be [2D, C] and w_out [M, D], D a multiple of 8")
        self.form, self.dtype, self.b_in, self.b_out = form, dtype, b_in, b_out
        self.w_in, self.w_out = self._codes(w_in), self._codes(w_out)
        self.state = torch.zeros((slots, self.D), dtype=torch.float32, device=w_in.device)

    @property
    def state(self) -> torch.Tensor:
        """The pool [slots, D]: read and written in place, or set (copied)."""
        return self._state

    @state.setter
    def state(self, value: torch.Tensor):
        # a row more, always zero: prefill's idle rows start and end there
        self._rows = torch.zeros((value.shape[0] + 1, self.D), dtype=torch.float32, device=value.device)
        self._state = self._rows[:-1]
        self._state.copy_(value)

    @staticmethod
    def _codes(w):
        q = torch.empty((w.shape[0], bc.i8_pitch(w.shape[1])), dtype=torch.int8, device=w.device)
        return bc.quantize_i8(w.contiguous(), q, torch.empty(w.shape[0], dtype=torch.float32, device=w.device))

    def _new(self, *shape):
        return torch.empty(shape, dtype=self.dtype, device=self.state.device)

    def prefill(self, x: torch.Tensor, slots: torch.Tensor, lengths: torch.Tensor | None = None,
                layout: int = bc.BC_TOKENS, fresh: bool = True):
        """Prompts x [N, T, C] (or maps [N, C, T]) of sequences slots [N] (distinct,
        but for idle rows) -> z [N, T, M] (or [N, M, T]); their rows of the pool
        take the states at each one's length.  fresh: from zero states, otherwise
        from the pool's."""
        D, N = self.D, x.shape[0]
        tokens = layout == bc.BC_TOKENS
        T = x.shape[1] if tokens else x.shape[2]
        bc._need(slots, (N,), (torch.int32, torch.int64), "prefill", "slots")
        bc._need(lengths, (N,), torch.int32, "prefill", "lengths")
        shape = (lambda c: (N, T, c)) if tokens else (lambda c: (N, c, T))
        p = bc.pointwise_mix_i8(*self.w_in, x, self._new(*shape(2 * D)), layout=layout, bias=self.b_in)
        gate, v = (p[..., :D], p[..., D:]) if tokens else (p[:, :D], p[:, D:])
        # an idle row is a sequence of no steps in the pool's extra row: no steps
        # leave that zero, whichever of several idle rows is stored last
        S, rows = self._state.shape[0], slots.long()
        idle = (rows < 0) | (rows >= S)
        rows = rows.masked_fill(idle, S)
        if lengths is None:
            lengths = torch.full((N,), T, dtype=torch.int32, device=x.device)
        lengths = lengths.masked_fill(idle, 0)
        h = torch.empty((N, D), dtype=torch.float32, device=x.device) if fresh else self._rows[rows]
        y = bc.gated_scan_fwd(gate, v, self._new(*shape(D)), h0=None if fresh else h, h_last=h, lengths=lengths,
                              form=self.form, layout=layout)
        self._rows[rows] = h
        return bc.pointwise_mix_i8(*self.w_out, y, self._new(*shape(self.M)), layout=layout, bias=self.b_out)

    def step(self, x: torch.Tensor, slots: torch.Tensor | None = None):
        """One token x [N, C] of each of N sequences (slots [N] int32, or None:
        the pool's first N rows) -> z [N, M]; the pool is updated."""
        D, N = self.D, x.shape[0]
        p = bc.pointwise_mix_i8(*self.w_in, x, self._new(N, 2 * D), bias=self.b_in)
        y = bc.gated_scan_step(p[:, :D], p[:, D:], self._state, self._new(N, D), slots=slots, form=self.form)
        return bc.pointwise_mix_i8(*self.w_out, y, self._new(N, self.M), bias=self.b_out)
