"""Linear attention with a decay for each head against its 64-bit oracle: the
chunked forward and backward, and the step.

Tolerances are counted, not measured: units of 2^-24 of each value's magnitude
(oracle/attention_oracle.py) and half a step of the output's type."""
import sys

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_1906_11367_amd import boxconv as bc

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FORM = {"logit": bc.BC_GATE_LOGIT, "log": bc.BC_GATE_LOG}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def check(name, got, want, mag, units, dt):
    g = to64(got)
    bound = units * A.EPS * mag + A.HALF_STEP[dt] * np.abs(want) * (1 + 2.0 ** -7) + 1e-37
    err = np.abs(g - want)
    assert np.isfinite(g).all(), name
    worst = (err / bound).max() if err.size else 0.0
    say(f"{name}: {worst:.3f} of the bound")
    assert worst <= 1.0, (name, worst, np.unravel_index((err / bound).argmax(), err.shape))


def gates(seed, form, *shape):
    """Memories from a step to thousands, with resets."""
    g = rand(seed, *shape) * 2 + 2
    if form == "log":
        g = torch.nn.functional.logsigmoid(g)
    g[torch.rand(shape, generator=torch.Generator().manual_seed(seed + 1)) < 0.02] = -float("inf")
    return g


class Case:
    """Inputs on the GPU and in 64 bits, of one seed."""

    def __init__(self, N, T, H, Dk, Dv, dt="f32", form="logit", heads=None, lengths=None, start=False, gate_f32=False,
                 heads_first=False, pad=0, fixed=False, seed=1):
        self.N, self.T, self.H, self.Dk, self.Dv, self.dt, self.form = N, T, H, Dk, Dv, dt, form
        Hq, Hk, Hv = heads or (H, H, H)
        self.scale = Dk ** -0.5
        self.heads_first, self.pad = heads_first, pad
        t = DT[dt]
        cpu = [rand(seed + i, N, T, h, d).to(t) for i, (h, d) in enumerate(((Hq, Dk), (Hk, Dk), (Hv, Dv), (H, Dv)))]
        gate = (-torch.exp2(-torch.arange(H, dtype=torch.float32)) if fixed else gates(seed + 9, form, N, T, H))
        gate = gate if gate_f32 or fixed else gate.to(t)
        s0 = rand(seed + 5, N, H, Dk, Dv) if start else None
        ds = rand(seed + 6, N, H, Dk, Dv) if start else None
        self.ref = A.attention(*(to64(v) for v in cpu[:3]), to64(gate.expand(N, T, H)), form, self.scale,
                               None if s0 is None else to64(s0), lengths, to64(cpu[3]), None if ds is None else to64(ds))
        if lengths is not None:   # what lies past an end is never looked at
            for n, ln in enumerate(lengths):
                for v in cpu:
                    v[n, max(ln, 0):] = float("nan")
                if not fixed:
                    gate[n, max(ln, 0):] = float("nan")
        self.q, self.k, self.v, self.dy = (self.place(v) for v in cpu)
        self.gate = gate.cuda()
        self.s0, self.ds = (None if v is None else v.cuda() for v in (s0, ds))
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.y = self.place(torch.full((N, T, H, Dv), 7.0, dtype=t))
        self.s_last = torch.full((N, H, Dk, Dv), 7.0, device="cuda")
        self.dq, self.dk, self.dv = (torch.empty_strided(v.shape, v.stride(), dtype=t, device="cuda").fill_(7)
                                     for v in (self.q, self.k, self.v))
        self.dgate = None if fixed else torch.full((N, T, H), 7.0, dtype=gate.dtype, device="cuda")
        self.ds0 = torch.full((N, H, Dk, Dv), 7.0, device="cuda")
        self.states = bc.linear_attention_states(N, T, H, Dk, Dv)

    def place(self, v):
        """On the GPU in the case's layout: heads outermost, or rows with a gap."""
        v = v.cuda()
        if self.heads_first:
            return v.transpose(1, 2).contiguous().transpose(1, 2)
        if self.pad:
            N, T, H, D = v.shape
            rows = torch.zeros((N, T, H * D + self.pad), dtype=v.dtype, device="cuda")
            rows[..., :H * D] = v.flatten(2)
            return rows[..., :H * D].unflatten(2, (H, D))
        return v

    def how(self):
        return dict(lengths=self.lengths, form=FORM[self.form], scale=self.scale)

    def forward(self, **kw):
        bc.linear_attention_fwd(self.q, self.k, self.v, self.gate, self.y, s0=self.s0, s_last=self.s_last,
                                states=self.states, **self.how(), **kw)

    def backward(self, **kw):
        bc.linear_attention_bwd(self.q, self.k, self.v, self.gate, self.states, self.dy, self.dq, self.dk, self.dv,
                                self.dgate, grad_s_last=self.ds, grad_s0=self.ds0, **self.how(), **kw)

    def check(self, names=("y", "s_last", "dq", "dk", "dv", "dgate", "ds0")):
        u = A.attention_units(self.T, self.Dk, self.Dv, self.dt)
        torch.cuda.synchronize()
        for name in names:
            got = getattr(self, name)
            if got is None:
                continue
            units, dt = u, self.dt
            if name in ("dq", "dk", "dv"):
                units += 16                       # heads that share
            if name == "dgate":
                units, dt = 2 * u + 16, "f32" if got.dtype is torch.float32 else self.dt
            if name in ("s_last", "ds0"):
                dt = "f32"
            check(name, got, *self.ref[name], units, dt)


CASES = [
    dict(N=1, T=1, H=1, Dk=1, Dv=1), dict(N=2, T=1, H=3, Dk=64, Dv=64, dt="bf16", start=True),
    dict(N=2, T=2, H=1, Dk=8, Dv=5, start=True), dict(N=1, T=15, H=2, Dk=7, Dv=16, dt="bf16"),
    dict(N=2, T=31, H=2, Dk=64, Dv=64, form="log"), dict(N=1, T=32, H=2, Dk=64, Dv=128, start=True),
    dict(N=1, T=33, H=2, Dk=128, Dv=64), dict(N=2, T=63, H=2, Dk=64, Dv=64, dt="bf16", form="log"),
    dict(N=1, T=64, H=2, Dk=128, Dv=64, dt="bf16", start=True), dict(N=1, T=65, H=2, Dk=64, Dv=128, dt="bf16"),
    dict(N=1, T=65, H=1, Dk=128, Dv=128), dict(N=1, T=127, H=2, Dk=40, Dv=72, dt="bf16", heads_first=True),
    dict(N=2, T=128, H=2, Dk=33, Dv=128, dt="bf16", start=True, lengths=[128, 0]),
    dict(N=3, T=129, H=2, Dk=64, Dv=64, start=True, lengths=[129, 64, 1]),
    dict(N=4, T=200, H=4, Dk=16, Dv=24, dt="bf16", heads=(4, 2, 1), lengths=[-3, 200, 500, 65], start=True),
    dict(N=2, T=150, H=6, Dk=20, Dv=12, heads=(2, 1, 3), start=True, pad=3),
    dict(N=1, T=260, H=2, Dk=128, Dv=128, dt="bf16", start=True, gate_f32=True),
    dict(N=1, T=300, H=3, Dk=65, Dv=127, dt="bf16", pad=5, form="log"),
    dict(N=1, T=300, H=3, Dk=127, Dv=65, pad=1, start=True, lengths=[257]),
    dict(N=2, T=400, H=2, Dk=64, Dv=32, fixed=True, form="log", heads_first=True),
    dict(N=1, T=700, H=2, Dk=32, Dv=32, dt="bf16", fixed=True, form="log", start=True, lengths=[600]),
    # one head, many spans and segments
    dict(N=1, T=3000, H=1, Dk=16, Dv=8, start=True), dict(N=1, T=2500, H=1, Dk=8, Dv=16, dt="bf16", start=True, lengths=[2111]),
    # more heads than blocks the card holds at once: one segment, spans all the same
    dict(N=40, T=257, H=16, Dk=4, Dv=4, dt="bf16", start=True),
    dict(N=9, T=1030, H=64, Dk=3, Dv=4, start=True),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda kw: "-".join(f"{v}" for v in kw.values()).replace(" ", ""))
def test_against_the_oracle(kw):
    say(kw)
    c = Case(**kw)
    c.forward()
    c.check(("y", "s_last"))
    c.backward()
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 600])
@pytest.mark.parametrize("D", [5, 64])
def test_the_first_gate_of_a_sequence_without_a_state(dt, T, D):
    """a_0 scales a state of zeros: its gradient is zero, not a rounding error."""
    c = Case(3, T, 2, D, D, dt, lengths=[T, 1, 0])
    c.forward()
    c.backward()
    assert (c.dgate[:, 0] == 0).all() and (T == 1 or (c.dgate[0, 1] != 0).any())
    c.check()
    # the same of a state that is given and is zero; of one that is not, only there
    c.s0 = torch.zeros((3, 2, D, D), device="cuda")
    c.s0[0, 1, D - 1, D - 1] = 1.0
    c.forward()
    c.backward()
    assert (c.dgate[1:, 0] == 0).all() and (c.dgate[0, 0, 0] == 0) and c.dgate[0, 0, 1] != 0


@pytest.mark.parametrize("dt,D", [("f32", 4), ("bf16", 8)])
def test_segments_of_many_chunks(dt, D):
    """Heads enough for segments of 2048 tokens, without kept states of all 2113: what is
    made for 32 chunks at a time is made again within a segment, and sequences end
    before, at and after such a place."""
    say(dt)
    c = Case(8, 2113, 64, D, D, dt, start=True, lengths=[2113, 2048, 1025, 1024, 1023, 0, 1500, 33])
    c.forward()
    c.check(("y", "s_last"))
    c.backward()
    c.check()
    c.states = None
    c.y.fill_(float("nan"))
    c.forward()
    c.check(("y", "s_last"))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_without_kept_states_and_optional_outputs(dt):
    """Inference: the same outputs without states, last state or lengths."""
    c = Case(1, 900, 2, 64, 64, dt, start=True)
    c.forward()
    y = c.y.clone()
    c.y.fill_(7)
    bc.linear_attention_fwd(c.q, c.k, c.v, c.gate, c.y, s0=c.s0, **c.how())
    assert torch.equal(c.y, y)
    c.check(("y",))
    c.backward()
    dq, dv = c.dq.clone(), c.dv.clone()
    bc.linear_attention_bwd(c.q, c.k, c.v, c.gate, c.states, c.dy, c.dq, c.dk, c.dv, None, grad_s_last=c.ds, **c.how())
    assert torch.equal(c.dq, dq) and torch.equal(c.dv, dv)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [100, 1500])
def test_state_in_place_of_the_initial_one(dt, T):
    """s_last in s0's memory, grad_s0 in grad_s_last's."""
    c = Case(1, T, 1, 32, 16, dt, start=True)
    c.s_last, c.ds0 = c.s0, c.ds
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_resets_everywhere(dt):
    """No decay leaves anything: every token sees itself alone, exactly, and the
    gates have no gradient."""
    c = Case(2, 150, 2, 16, 16, dt, start=True)
    c.gate.fill_(-float("inf"))
    c.forward()
    c.backward()
    q, k, v = (to64(t) for t in (c.q, c.k, c.v))
    own = c.scale * (q * k).sum(-1, keepdims=True) * v
    mag = c.scale * (np.abs(q) * np.abs(k)).sum(-1, keepdims=True) * np.abs(v)
    check("y", c.y, own, mag, A.attention_units(1, 16, 16, dt), dt)
    last = k[:, -1, :, :, None] * v[:, -1, :, None, :]
    check("s_last", c.s_last, last, np.abs(last), 8, "f32")
    assert (c.dgate == 0).all() and (c.ds0 == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("inf"), 90.0, 3e38])
def test_decays_of_one(dt, value):
    """sigmoid(gate) = 1: the plain running sum; its gate has no slope."""
    c = Case(1, 200, 1, 8, 8, dt)
    c.gate.fill_(value)
    c.ref = A.attention(*(to64(t) for t in (c.q, c.k, c.v)), np.full((1, 200, 1), 700.0), "logit", c.scale, dy=to64(c.dy))
    c.forward()
    c.backward()
    c.check(("y", "s_last", "dq", "dk", "dv"))
    assert (c.dgate.float().abs() <= 1e-30).all()


def test_a_reset_keeps_precision_after_it():
    """Decays within a chunk that holds resets: the exponents' sums are taken in
    64 bits, so a reset's 10^4 does not cost the others their digits."""
    c = Case(1, 64, 1, 4, 4, "f32", form="log")
    g = torch.full((1, 64, 1), -0.01)
    g[0, 5::7] = -float("inf")
    c.gate.copy_(g)
    c.ref = A.attention(*(to64(t) for t in (c.q, c.k, c.v)), to64(g), "log", c.scale, dy=to64(c.dy))
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_non_finite_values_stay_in_their_sequence_and_head(dt):
    clean = Case(2, 140, 3, 16, 16, dt, start=True)
    clean.forward()
    clean.backward()
    c = Case(2, 140, 3, 16, 16, dt, start=True)
    for t, v in ((c.q, float("nan")), (c.k, float("inf")), (c.v, -float("inf")), (c.dy, float("nan"))):
        t[1, 70, 2, 3] = v
    c.gate[1, 71, 2] = float("nan")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for name in ("y", "s_last", "dq", "dk", "dv", "dgate", "ds0"):
        a, b = getattr(c, name).clone(), getattr(clean, name).clone()
        at = (1, 2) if name in ("s_last", "ds0") else (1, slice(None), 2)
        a[at], b[at] = 0, 0
        assert torch.equal(a, b), name


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_shared_memory_as_an_input(dt):
    """Keys expanded over heads and queries over tokens (strides of zero)."""
    N, T, H, D = 2, 100, 3, 16
    k1, q1 = rand(1, N, T, 1, D).to(DT[dt]).cuda(), rand(2, N, 1, H, D).to(DT[dt]).cuda()
    k, q = k1.expand(N, T, H, D), q1.expand(N, T, H, D)
    v, gate = rand(3, N, T, H, D).to(DT[dt]).cuda(), gates(4, "logit", N, T, H).to(DT[dt]).cuda()
    y = [torch.empty((N, T, H, D), dtype=DT[dt], device="cuda") for _ in range(2)]
    bc.linear_attention_fwd(q, k, v, gate, y[0])
    bc.linear_attention_fwd(q.contiguous(), k.contiguous(), v, gate, y[1])
    assert torch.equal(y[0], y[1])


def test_slices_of_one_projection_and_rows_beyond():
    """q, k, v and the gate out of one buffer's rows, the gradients into one; what
    lies between and around them stays as it was."""
    N, T, H, D = 2, 90, 2, 32
    W = 3 * H * D + 8
    rows = rand(1, N, T, W).to(torch.bfloat16).cuda()
    cut = lambda b: [b[..., i * H * D:(i + 1) * H * D].unflatten(2, (H, D)) for i in range(3)]
    gate_of = lambda b: b[..., 3 * H * D:3 * H * D + H]
    q, k, v = cut(rows)
    out = torch.full((N, T + 2, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    grads = torch.full((N, T, W), 7.0, dtype=torch.bfloat16, device="cuda")
    y, states, dy = out[:, 1:T + 1], bc.linear_attention_states(N, T, H, D, D), rand(2, N, T, H, D).to(torch.bfloat16).cuda()
    bc.linear_attention_fwd(q, k, v, gate_of(rows), y, states=states)
    bc.linear_attention_bwd(q, k, v, gate_of(rows), states, dy, *cut(grads), gate_of(grads))
    ref = A.attention(*(to64(t) for t in (q, k, v)), to64(gate_of(rows)), "logit", 1.0, dy=to64(dy))
    u = A.attention_units(T, D, D, "bf16")
    check("y", y, *ref["y"], u, "bf16")
    for name, got in zip(("dq", "dk", "dv"), cut(grads)):
        check(name, got, *ref[name], u + 16, "bf16")
    check("dgate", gate_of(grads), *ref["dgate"], 2 * u + 16, "bf16")
    assert (out[:, 0] == 7).all() and (out[:, -1] == 7).all() and (grads[..., 3 * H * D + H:] == 7).all()


def test_bits_are_the_same_every_time_and_on_other_streams():
    c = Case(2, 900, 4, 64, 64, "bf16", heads=(2, 4, 1), start=True)
    c.forward()
    c.backward()
    first = {n: getattr(c, n).clone() for n in ("y", "s_last", "dq", "dk", "dv", "dgate", "ds0")}
    d = Case(2, 900, 4, 64, 64, "bf16", heads=(2, 4, 1), start=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, case in zip(streams, (c, d)):
        with torch.cuda.stream(s):
            case.forward()
            case.backward()
    torch.cuda.synchronize()
    for n, v in first.items():
        assert torch.equal(getattr(c, n), v) and torch.equal(getattr(d, n), v), n


def test_under_a_graph():
    """Forward, backward and a step captured once, replayed on other inputs."""
    N, T, H, D = 2, 700, 2, 64
    c = Case(N, T, H, D, D, "bf16", heads=(2, 1, 2), start=True)
    sizes = (N, T, H, 2, 1, 2, D, D, bc.BC_BF16)
    ws = torch.empty(max(bc.linear_attention_workspace_bytes(op, *sizes) for op in (0, 1)), dtype=torch.uint8, device="cuda")
    pool, y1 = torch.zeros((4, H, D, D), device="cuda"), torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")

    def all_of_it(ws):
        c.forward(ws=ws)
        c.backward(ws=ws)
        bc.linear_attention_step(c.q[:, 0], c.k[:, 0], c.v[:, 0], c.gate[:, 0], pool, y1, slots=slots, scale=c.scale)

    names = ("y", "s_last", "dq", "dk", "dv", "dgate", "ds0")
    all_of_it(ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        all_of_it(ws)
    for seed in (11, 12, 13):
        for i, t in enumerate((c.q, c.k, c.v, c.dy)):
            t.copy_(rand(seed + 10 * i, *t.shape))
        pool.fill_(seed)
        all_of_it(None)
        eager = [getattr(c, n).clone() for n in names] + [pool.clone(), y1.clone()]
        for n in names:
            getattr(c, n).zero_()
        pool.fill_(seed)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, [getattr(c, n) for n in names] + [pool, y1]):
            assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """Sequences 2^31 and more elements apart, and a pool of more than 2^32."""
    N, T, H, D = 2, 70, 1, 64
    far = 2 ** 31 + 24
    buf = torch.zeros(far + T * 3 * D, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(buf, (N, T, 3 * D), (far, 3 * D, 1))
    rows.copy_(rand(1, N, T, 3 * D))
    q, k, v = (rows[..., i * D:(i + 1) * D].unflatten(2, (H, D)) for i in range(3))
    gate = gates(2, "logit", N, T, H).cuda()
    y = [torch.empty((N, T, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bc.linear_attention_fwd(q, k, v, gate, y[0])
    bc.linear_attention_fwd(q.contiguous(), k.contiguous(), v.contiguous(), gate, y[1])
    assert torch.equal(*y) and y[0].abs().max() > 0
    del buf, rows, q, k, v
    S = 2 ** 32 // (16 * 128 * 128) + 3
    pool = torch.empty((S, 16, 128, 128), device="cuda")
    pool[S - 1] = 1.0
    one = torch.ones((1, 16, 128), dtype=torch.bfloat16, device="cuda")
    y1 = torch.empty_like(one)
    bc.linear_attention_step(one, one, one, torch.full((1, 16), float("inf"), device="cuda"), pool, y1,
                             slots=torch.tensor([S - 1], dtype=torch.int32, device="cuda"))
    assert (pool[S - 1] == 2).all() and (y1 == 256).all()


# ---- the step -----------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,heads,Dk,Dv,form", [
    (1, 1, (1, 1, 1), 1, 1, "logit"), (3, 2, (1, 2, 2), 64, 64, "logit"), (5, 4, (4, 1, 2), 33, 45, "log"),
    (40, 16, (16, 16, 16), 128, 128, "log"), (7, 6, (2, 3, 6), 100, 20, "logit"), (70, 3, (3, 3, 1), 5, 127, "logit")])
@pytest.mark.parametrize("place", ["in place", "beside"])
def test_step(dt, N, H, heads, Dk, Dv, form, place):
    """Slots in any order, idle rows, states that no row names."""
    t, S = DT[dt], N + 3
    q, k, v = (rand(i, N, h, d).to(t).cuda() for i, (h, d) in enumerate(zip(heads, (Dk, Dk, Dv))))
    gate, state = gates(5, form, N, H).to(t).cuda(), rand(6, S, H, Dk, Dv).cuda()
    slots = torch.randperm(S, generator=torch.Generator().manual_seed(N))[:N].to(torch.int32)
    if N > 2:
        slots[1], slots[N - 1] = -1, S
    before, slots_np = to64(state), slots.numpy()
    live = (slots_np >= 0) & (slots_np < S)
    out = state if place == "in place" else torch.full_like(state, 7.0)
    y = torch.full((N, H, Dv), 7.0, dtype=t, device="cuda")
    bc.linear_attention_step(q, k, v, gate, state, y, slots=slots.cuda(), state_out=None if place == "in place" else out,
                             form=FORM[form], scale=0.5)
    at = np.where(live, slots_np, 0)
    wy, my, ws, ms = A.step(to64(q), to64(k), to64(v), to64(gate), form, 0.5, before[at])
    u = Dk + 64
    check("y", y[torch.from_numpy(live).cuda()], wy[live], my[live], u, dt)
    check("state", out[torch.from_numpy(at[live]).cuda()], ws[live], ms[live], 64, "f32")
    assert (y[torch.from_numpy(~live).cuda()] == 0).all()
    rest = np.setdiff1d(np.arange(S), at[live])
    assert (to64(out)[rest] == (before[rest] if place == "in place" else 7.0)).all()
    if place == "beside":
        assert (to64(state) == before).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_steps_follow_a_prompt(dt):
    """A prompt, then single tokens on its state, against the whole sequence."""
    N, T, H, D, P = 2, 90, 2, 32, 83
    c = Case(N, T, H, D, D, dt, heads=(2, 1, 2))
    pool = torch.zeros((N, H, D, D), device="cuda")
    bc.linear_attention_fwd(c.q[:, :P], c.k[:, :P], c.v[:, :P], c.gate[:, :P], c.y[:, :P], s_last=pool, **c.how())
    for t in range(P, T):
        y = torch.empty((N, H, D), dtype=DT[dt], device="cuda")
        bc.linear_attention_step(c.q[:, t], c.k[:, t], c.v[:, t], c.gate[:, t], pool, y, form=FORM[c.form], scale=c.scale)
        c.y[:, t] = y
    c.s_last = pool
    c.check(("y", "s_last"))


def test_calls_of_one_layout():
    """Layouts are checked when they are met first: later calls of the same layout take
    their own tensors, numbers and pointers, and another layout is checked again."""
    N, H, D = 2, 3, 16
    mk = lambda seed: torch.randn(N, H, D, generator=torch.Generator().manual_seed(seed)).cuda()
    q, k, v, y = mk(1), mk(2), mk(3), torch.empty(N, H, D, device="cuda")
    g, pool = torch.zeros(N, H, device="cuda"), torch.zeros(N, H, D, D, device="cuda")
    scale = torch.tensor(1.0)
    one = bc.linear_attention_step(q, k, v, g, pool, y, scale=scale).clone()
    scale.fill_(2.0)
    pool.zero_()
    # (the same tensor for scale, another value; another q in the same place)
    assert torch.equal(bc.linear_attention_step(q, k, v, g, pool, y, scale=scale), 2 * one)
    pool.zero_()
    q.mul_(-1)
    assert torch.equal(bc.linear_attention_step(q, k, v, g, pool, y, scale=1.0), -one)
    with pytest.raises(bc.BoxConvError):      # a view that starts off the vectors' alignment
        flat = torch.zeros(N * H * D + 1, device="cuda")
        bc.linear_attention_step(flat[1:].view(N, H, D), k, v, g, pool, y)
    with pytest.raises(bc.BoxConvError):      # of the same shape, rows in another order
        bc.linear_attention_step(q, k, v, g, torch.zeros(N, D, H, D, device="cuda").transpose(1, 2), y)
    with pytest.raises(bc.BoxConvError):
        bc.linear_attention_step(q.cpu(), k, v, g, pool, y)


# ---- rows that end inside a lane's columns --------------------------------------

# fp32 rows of 65 to 128 elements that are whole vectors of 4 and not of the 8 columns a lane has
HALF_ROWS = [dict(N=2, T=70, H=3, Dk=64, Dv=68), dict(N=1, T=90, H=2, Dk=100, Dv=32, start=True),
             dict(N=2, T=65, H=3, Dk=124, Dv=92, form="log", lengths=[65, 40]), dict(N=1, T=900, H=2, Dk=76, Dv=84, start=True),
             dict(N=2, T=40, H=6, Dk=108, Dv=116, heads=(2, 3, 1), start=True)]


@pytest.mark.parametrize("layout", ["tokens", "heads", "slices"])
@pytest.mark.parametrize("kw", HALF_ROWS, ids=lambda kw: "-".join(f"{v}" for v in kw.values()).replace(" ", ""))
def test_rows_that_end_inside_a_lanes_columns(kw, layout):
    """Every output is the oracle's, and nothing beside a row is written: in `slices` the
    rows of y, and of the gradients in one buffer, stand between gaps."""
    say(kw, layout)
    c = Case(**kw, heads_first=layout == "heads")
    N, T, H = c.N, c.T, c.H
    if layout == "slices":
        parts = [(c.q.shape[2], c.Dk), (c.k.shape[2], c.Dk), (c.v.shape[2], c.Dv), (H, c.Dv)]
        width = sum(h * (d + 4) for h, d in parts)
        rows, known = (torch.full((N, T, width), 7.0, device="cuda") for _ in range(2))
        at = 0
        for name, (h, d) in zip(("dq", "dk", "dv", "y"), parts):
            cut = lambda t: t[..., at:at + h * (d + 4)].unflatten(2, (h, d + 4))[..., :d]
            setattr(c, name, cut(rows))
            cut(known).fill_(8.0)
            at += h * (d + 4)
    c.forward()
    c.check(("y", "s_last"))
    c.backward()
    c.check()
    if layout == "slices":
        assert (rows[known == 7.0] == 7.0).all()


@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_a_neighbouring_row_is_not_looked_at(layout):
    """Non-finite values of one head, in rows that end inside a lane's columns, leave the others' bits."""
    names = ("y", "s_last", "dq", "dk", "dv", "dgate", "ds0")
    cases = [Case(2, 70, 3, 68, 100, start=True, heads_first=layout == "heads") for _ in range(2)]
    c = cases[1]
    for t in (c.q, c.k, c.v, c.dy):
        t[1, :, 1] = float("nan")
        t[0, 33, 2] = float("inf")
    for x in cases:
        x.forward()
        x.backward()
    torch.cuda.synchronize()
    for name in names:
        a, b = (getattr(x, name).clone() for x in cases)
        a, b = (t if name in ("s_last", "ds0") else t.transpose(1, 2) for t in (a, b))
        for n, h in ((0, 0), (0, 1), (1, 0), (1, 2)):
            assert torch.equal(a[n, h], b[n, h]), (name, n, h)


# ---- decays above one -----------------------------------------------------------

def growing(kind, T, zero_k, zero_dy):
    """Logarithms of decays [T], those of no run of up to 32 tokens summing to more than 60 log 2;
    zero_k, zero_dy: tokens whose keys, or output gradients, are zero, so that neither
    states nor their gradients grow past 2^60."""
    g = torch.full((T,), -0.1)
    if kind == "blocks":            # e^40 between two resets: empty states, then ones whose gradient is empty
        for b in range(0, T - 11, 12):
            g[b], g[b + 1:b + 11] = -float("inf"), 4.0
            zero_k[b:b + 6] = True
            zero_dy[b + 6:b + 12] = True
    elif kind == "from 1e-30":      # a start state that e^38 brings to 1e-13
        g[:19] = 2.0
        zero_k[:18] = True
        zero_dy[5:] = True
    elif kind == "segments":        # e^160 in a segment of 128 tokens, over states of zeros
        g[:1024], g[1024] = 1.25, -float("inf")
        zero_k[:1024] = True
        zero_dy[20:1024] = True
    elif kind == "slowly":          # e^60 over many chunks, from 1e-30
        g[:] = 0.3
        zero_k[:T - 30] = True
        zero_dy[20:] = True
    else:                           # up and down
        g = 0.6 * rand(77, T)
    return g


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv,heads", [(64, 64, None), (128, 96, (1, 2, 2)), (7, 5, None), (100, 128, (2, 1, 1))])
@pytest.mark.parametrize("kind,N,T,start", [("blocks", 1, 96, 0.0), ("from 1e-30", 1, 50, 1e-30), ("segments", 8, 2048, 0.0),
                                            ("slowly", 1, 200, 1e-30), ("random", 1, 130, 1.0)])
def test_decays_above_one(kind, N, T, start, Dk, Dv, heads, dt):
    """Outputs and gradients are the recurrence's, also where a segment's decays together
    pass fp32's range."""
    say(kind, T, Dk, Dv, dt)
    if N > 1:
        Dk, Dv = min(Dk, 8), min(Dv, 8)
    c = Case(N, T, 2, Dk, Dv, dt, form="log", heads=heads, start=True, gate_f32=True)
    zero_k, zero_dy = torch.zeros((2, T), dtype=torch.bool)
    c.gate.copy_(growing(kind, T, zero_k, zero_dy)[None, :, None].expand(N, T, 2))
    c.k[:, zero_k.cuda()] = 0
    c.dy[:, zero_dy.cuda()] = 0
    c.s0 *= start
    if start != 1.0:
        c.ds *= 0
    c.ref = A.attention(*(to64(t) for t in (c.q, c.k, c.v)), to64(c.gate), "log", c.scale, to64(c.s0), None, to64(c.dy),
                        to64(c.ds))
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    # a factor 2^x of a score has its exponent to 2^-24 of itself: 60 log 2 units more
    u = A.attention_units(T, Dk, Dv, dt) + 48
    for name in ("y", "dq", "dk", "dv"):
        check(name, getattr(c, name), *c.ref[name], u + 16, dt)
    for name in ("s_last", "ds0", "dgate"):
        check(name, getattr(c, name), *c.ref[name], u if name != "dgate" else 2 * u + 16, "f32")


# ---- sizes of errors, beside their bounds ----------------------------------------

NORMS = [dict(N=1, T=260, H=2, Dk=128, Dv=128), dict(N=2, T=300, H=2, Dk=64, Dv=96, form="log"), dict(N=1, T=1100, H=1, Dk=128, Dv=64),
         dict(N=1, T=3000, H=1, Dk=16, Dv=32), dict(N=40, T=257, H=8, Dk=24, Dv=20)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kw", NORMS, ids=lambda kw: "-".join(f"{v}" for v in kw.values()))
def test_the_gates_gradients_as_a_whole(kw, dt):
    """Worst cases add up over thousands of tokens; roundings do not.  Those of a product
    q . dq are independent and come to u of the product: u = 2^-16 / sqrt(3) in bf16 (a score
    or a state in two parts, off by at most 2^-16, any size below as likely), 2^-24 sqrt(terms)
    in fp32; those of a sum over tokens to the root of the sum of squares."""
    c = Case(**kw, dt=dt, start=True, gate_f32=True)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    u = 2.0 ** -16 / 3 ** 0.5 if dt == "bf16" else 2.0 ** -24 * (c.Dk + c.Dv + 64) ** 0.5
    q, k, gate = to64(c.q), to64(c.k), to64(c.gate)
    squares = (q * c.ref["dq"][0]).sum(-1) ** 2 + (k * c.ref["dk"][0]).sum(-1) ** 2
    edge = (to64(c.s_last) * to64(c.ds)).sum((2, 3))[:, None] ** 2
    slope = 1.0 / (1.0 + np.exp(np.minimum(gate, 700.0))) if c.form == "logit" else 1.0
    bound = np.linalg.norm(u * slope * np.sqrt(squares[:, ::-1].cumsum(1)[:, ::-1] + edge))
    want = c.ref["dgate"][0]
    err, size = np.linalg.norm(to64(c.dgate) - want), np.linalg.norm(want)
    say(f"{err / size:.2e}, bound {bound / size:.2e}")
    assert err <= bound and bound <= (1e-3 if dt == "bf16" else 1e-4) * size


@pytest.mark.parametrize("kw", NORMS, ids=lambda kw: "-".join(f"{v}" for v in kw.values()))
def test_states_of_bf16_operands_are_fp32(kw):
    """What a state takes in is a sum of three bf16 parts: a decay's 4 units of 2^-24, the
    parts' and the product's one each, and roundings of sums over at most some hundred
    tokens that a state remembers, sqrt(100) / 2.  (In two parts 2^-16 / sqrt(3) at most: up to 148 units.)"""
    c = Case(**kw, dt="bf16", start=True, gate_f32=True)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for name in ("s_last", "ds0"):
        want = c.ref[name][0]
        err = np.linalg.norm(to64(getattr(c, name)) - want) / np.linalg.norm(want)
        say(f"{name}: {err / A.EPS:.1f} units")
        assert err <= 16 * A.EPS, name
