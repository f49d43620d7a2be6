"""The gated scan on the GPU against the step-by-step evaluation in 64 bits:
forward, backward and the single-token step.  The bars are the oracle's own
bounds on a 32-bit evaluation (oracle/recurrent_oracle.py), plus the rounding
of the outputs' type."""
import sys

import numpy as np
import pytest
import torch

from oracle import recurrent_oracle as R
from paper_1906_11367_amd import boxconv as bc

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LAYOUT = {"tokens": bc.BC_TOKENS, "maps": bc.BC_MAPS}
FORM = {"logit": bc.BC_GATE_LOGIT, "value": bc.BC_GATE_VALUE}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def shape_of(N, T, C, layout):
    return (N, T, C) if layout == "tokens" else (N, C, T)


def inputs(seed, N, T, C, dt, layout, form, packed=False):
    g = torch.Generator().manual_seed(seed)
    shape = shape_of(N, T, C, layout)
    gate = torch.randn(shape, generator=g) * 2 + 2
    reset = torch.rand(shape, generator=g) < 0.02
    gate = (torch.sigmoid(gate).masked_fill(reset, 0.0) * torch.sign(torch.rand(shape, generator=g) - 0.1)
            if form == "value" else gate.masked_fill(reset, -float("inf")))
    d = {"gate": gate, "x": torch.randn(shape, generator=g), "gy": torch.randn(shape, generator=g)}
    d = {k: v.to(DT[dt]).cuda() for k, v in d.items()}
    if packed:
        dim = 2 if layout == "tokens" else 1
        p = torch.cat([d["gate"], d["x"]], dim=dim)
        d["gate"], d["x"] = p.narrow(dim, 0, C), p.narrow(dim, C, C)
    d["h0"] = torch.randn((N, C), generator=g).cuda()
    d["gh"] = torch.randn((N, C), generator=g).cuda()
    return d


def close(got, want, bound, out_dt, what):
    """|got - want| within the 32-bit bound and the rounding of the output's type."""
    g = to64(got)
    if out_dt == "bf16":
        bound = bound + R.U_BF16 * (np.abs(want) + bound)
    else:
        bound = bound + R.EPS * np.abs(want)
    assert np.isfinite(g).all(), what
    over = np.abs(g - want) - bound
    worst = np.unravel_index(np.argmax(over), over.shape)
    assert over.max() <= 0, f"{what}: at {worst} got {g[worst]} want {want[worst]} bound {bound[worst]}"


def run_both(d, N, T, C, dt, layout, form, lengths=None, start=True, out_dt=None, packed_grad=False, ws_slack=0):
    """Forward and backward through the library, compared with the oracle."""
    out_dt = out_dt or dt
    shape = shape_of(N, T, C, layout)
    nan = float("nan")
    y = torch.full(shape, nan, dtype=DT[out_dt], device="cuda")
    h_last = torch.full((N, C), nan, device="cuda")
    states = bc.gated_scan_states(N, T, C, DT[dt], LAYOUT[layout]).fill_(nan)
    kw = dict(form=FORM[form], layout=LAYOUT[layout])
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    h0 = d["h0"] if start else None
    bc.gated_scan_fwd(d["gate"], d["x"], y, h0=h0, h_last=h_last, lengths=ln, states=states, **kw)
    if packed_grad:
        dim = 2 if layout == "tokens" else 1
        full = list(shape)
        full[dim] *= 2
        p = torch.full(full, nan, dtype=DT[out_dt], device="cuda")
        gg, gx = p.narrow(dim, 0, C), p.narrow(dim, C, C)
    else:
        gg, gx = (torch.full(shape, nan, dtype=DT[out_dt], device="cuda") for _ in range(2))
    gh0 = torch.full((N, C), nan, device="cuda")
    bc.gated_scan_bwd(d["gate"], d["x"], states, d["gy"], gg, gx, grad_h_last=d["gh"] if start else None, grad_h0=gh0,
                      lengths=ln, **kw)
    torch.cuda.synchronize()
    s = lambda v: R.seq(to64(v), layout)
    h0n = to64(d["h0"]) if start else None
    with np.errstate(invalid="ignore"):
        h, yy, e = R.scan_forward(s(d["gate"]), s(d["x"]), h0n, lengths, form)
        b = R.scan_backward(s(d["gate"]), s(d["x"]), s(d["gy"]), h0n, to64(d["gh"]) if start else None, lengths, form)
    close(y, R.unseq(yy, layout), R.unseq(e[1:], layout), out_dt, "y")
    close(h_last, h[T], e[T], "f32", "h_last")
    close(gx, R.unseq(b["x"], layout), R.unseq(b["x_bound"], layout), out_dt, "grad_x")
    close(gg, R.unseq(b["gate"], layout), R.unseq(b["gate_bound"], layout), out_dt, "grad_gate")
    close(gh0, b["h0"], b["h0_bound"], "f32", "grad_h0")
    if lengths is not None:   # zero past the end, exactly
        dead = torch.arange(T)[None, :] >= torch.tensor(lengths)[:, None]
        dead = (dead[:, :, None] if layout == "tokens" else dead[:, None, :]).expand(shape)
        for v in (y, gg, gx):
            assert (v.float().cpu()[dead] == 0).all()
    return y, h_last, gg, gx, gh0


# lengths around a lane's run (4, 8), a kept state (128) and a tile (256), and
# channel counts around a lane's (4, 8) and a block's (32, 64)
@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,C", [(1, 1, 1), (3, 2, 7), (2, 5, 8), (1, 127, 33), (2, 128, 64), (2, 129, 65),
                                   (1, 255, 130), (1, 257, 9), (5, 31, 100), (1, 1000, 72), (2, 513, 31), (3, 9, 300),
                                   (2, 17, 257), (2, 33, 70), (1, 64, 40), (2, 65, 66), (1, 256, 33)])
def test_tokens(N, T, C, dt, form):
    say("scan tokens", N, T, C, dt, form)
    run_both(inputs(11, N, T, C, dt, "tokens", form), N, T, C, dt, "tokens", form)


# a few steps of many channels: slabs of more channels than a block has lanes
@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,C", [(2, 1, 300), (3, 2, 513), (2, 3, 128), (2, 4, 256), (5, 5, 257), (1, 7, 1030),
                                   (3, 8, 640)])
def test_few_steps_of_many_channels(N, T, C, dt, form):
    say("scan few steps", N, T, C, dt, form)
    run_both(inputs(22, N, T, C, dt, "tokens", form), N, T, C, dt, "tokens", form)
    run_both(inputs(23, N, T, C, dt, "tokens", form), N, T, C, dt, "tokens", form, [T // 2] * N, start=False)


# few chains, long enough that the forward cuts them into longer tiles (256 steps)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,C,lengths", [(1, 16385, 9, None), (1, 16640, 64, [16639]), (2, 17001, 70, [17001, 4353]),
                                           (3, 16500, 3, [0, 1, 16257])])
def test_few_long_chains(N, T, C, lengths, dt):
    say("scan few long chains", N, T, C, lengths, dt)
    run_both(inputs(21, N, T, C, dt, "tokens", "logit"), N, T, C, dt, "tokens", "logit", lengths)


# lengths around a lane's run (8), a wave's segment (512) and several of them;
# rows that take one wave, four and sixteen
@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,C", [(1, 1, 1), (2, 7, 3), (3, 8, 5), (1, 511, 6), (2, 512, 4), (1, 513, 7),
                                   (2, 2049, 3), (1, 9000, 2), (9, 600, 130), (2, 520, 2100), (3, 4, 50),
                                   (2, 9, 70), (5, 32, 33), (2, 33, 17), (3, 64, 5), (2, 65, 9), (2, 128, 7), (2, 129, 3),
                                   (1, 256, 5), (3, 257, 3), (2, 17000, 3)])
def test_maps(N, T, C, dt, form):
    say("scan maps", N, T, C, dt, form)
    run_both(inputs(12, N, T, C, dt, "maps", form), N, T, C, dt, "maps", form)


@pytest.mark.parametrize("layout", ["tokens", "maps"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,lengths", [(300, [300, 0, 1, 299, 128, 129]), (700, [0, 700, 513, 512, 511, 8]),
                                       (5, [0, 0, 5, 4, 1, 3]), (30, [30, 0, 7, 8, 9, 29]), (100, [64, 0, 100, 65, 1, 99]), (300, [-4, 900, 256, 257, 255, 2])])
def test_ragged(T, lengths, dt, layout):
    """Sequences of their own lengths (out-of-range ones are clamped); what
    stands past them, NaN here, reaches nothing."""
    say("scan ragged", T, lengths, dt, layout)
    N, C = len(lengths), 37
    for form in ("logit", "value"):
        d = inputs(13, N, T, C, dt, layout, form)
        dead = torch.arange(T)[None, :] >= torch.tensor(lengths)[:, None]
        dead = (dead[:, :, None] if layout == "tokens" else dead[:, None, :]).cuda()
        for k in ("gate", "x", "gy"):
            d[k] = d[k].masked_fill(dead, float("nan"))
        run_both(d, N, T, C, dt, layout, form, lengths=lengths)


@pytest.mark.parametrize("layout", ["tokens", "maps"])
@pytest.mark.parametrize("dt,out_dt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_halves_of_one_projection(layout, dt, out_dt):
    """gate and x as the halves of one tensor, their gradients as the halves of
    another; bf16 outputs of fp32 inputs; no initial state."""
    N, T, C = 2, 264, 72
    d = inputs(14, N, T, C, dt, layout, "logit", packed=True)
    assert not d["gate"].is_contiguous()
    run_both(d, N, T, C, dt, layout, "logit", out_dt=out_dt, packed_grad=True, start=False)


@pytest.mark.parametrize("layout", ["tokens", "maps"])
def test_wide_strides(layout):
    """Rows and batches far apart, the gap between them full of NaN."""
    N, T, C = 3, 133, 40
    d = inputs(15, N, T, C, "f32", layout, "logit")
    shape = shape_of(N, T, C, layout)
    for k in ("gate", "x"):
        big = torch.full((N + 1, shape[1] + 3, shape[2] + 20), float("nan"), device="cuda")
        view = big[:N, :shape[1], :shape[2]]
        view.copy_(d[k])
        d[k] = view
    run_both(d, N, T, C, "f32", layout, "logit")


@pytest.mark.parametrize("layout", ["tokens", "maps"])
def test_split_sequences_continue(layout):
    """A sequence in two calls, the second from the first's last state, gives
    the states of one call (in the 32-bit bound); h_last may be h0's memory."""
    N, T, C, cut = 2, 700, 48, 300
    d = inputs(16, N, T, C, "f32", layout, "logit")
    dim = 1 if layout == "tokens" else 2
    part = lambda v, lo, n: v.narrow(dim, lo, n).contiguous()
    h = d["h0"].clone()
    ys = []
    for lo, n in ((0, cut), (cut, T - cut)):
        y = torch.empty(shape_of(N, n, C, layout), device="cuda")
        bc.gated_scan_fwd(part(d["gate"], lo, n), part(d["x"], lo, n), y, h0=h, h_last=h, layout=LAYOUT[layout])
        ys.append(y)
    hh, yy, e = R.scan_forward(R.seq(to64(d["gate"]), layout), R.seq(to64(d["x"]), layout), to64(d["h0"]))
    close(torch.cat(ys, dim=dim), R.unseq(yy, layout), R.unseq(e[1:], layout), "f32", "y")
    close(h, hh[T], e[T], "f32", "h_last")


@pytest.mark.parametrize("layout", ["tokens", "maps"])
def test_extreme_gates(layout):
    """Gates of both infinities and of the type's lowest and highest values:
    exact resets and exact holds, no NaN."""
    N, T, C = 1, 260, 16
    d = inputs(17, N, T, C, "f32", layout, "logit")
    low, high = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    g = torch.tensor([-float("inf"), low, float("inf"), high, 0.0, -90.0, 90.0, -200.0], device="cuda")
    pick = torch.randint(0, len(g), d["gate"].shape, generator=torch.Generator().manual_seed(3)).cuda()
    d["gate"] = g[pick]
    run_both(d, N, T, C, "f32", layout, "logit")


@pytest.mark.parametrize("layout", ["tokens", "maps"])
def test_non_finite_values_stay_in_their_channel(layout):
    N, T, C, t, c = 2, 600, 40, 301, 5
    d = inputs(18, N, T, C, "f32", layout, "logit")
    d["gate"] = d["gate"].clamp(min=-20)
    at = (0, t, c) if layout == "tokens" else (0, c, t)
    clean = torch.empty_like(d["x"])
    bc.gated_scan_fwd(d["gate"], d["x"], clean, h0=d["h0"], layout=LAYOUT[layout])
    for name in ("x", "gate"):
        bad = {k: v.clone() for k, v in d.items()}
        bad[name][at] = float("nan")
        y = torch.empty_like(clean)
        bc.gated_scan_fwd(bad["gate"], bad["x"], y, h0=d["h0"], layout=LAYOUT[layout])
        hit = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
        hit[(0, slice(t, None), c) if layout == "tokens" else (0, c, slice(t, None))] = True
        assert torch.isnan(y[hit]).all()
        assert torch.equal(y[~hit], clean[~hit])


def test_same_bits_every_time():
    """No sum depends on the order in which blocks run."""
    for layout, (N, T, C) in (("tokens", (2, 3000, 200)), ("maps", (2, 3000, 200))):
        d = inputs(19, N, T, C, "bf16", layout, "logit")
        first = None
        for _ in range(3):
            y, h = torch.empty_like(d["x"]), torch.empty((N, C), device="cuda")
            st = bc.gated_scan_states(N, T, C, torch.bfloat16, LAYOUT[layout])
            bc.gated_scan_fwd(d["gate"], d["x"], y, h0=d["h0"], h_last=h, states=st, layout=LAYOUT[layout])
            gg, gx, gh = torch.empty_like(y), torch.empty_like(y), torch.empty_like(h)
            bc.gated_scan_bwd(d["gate"], d["x"], st, d["gy"], gg, gx, grad_h_last=d["gh"], grad_h0=gh,
                              layout=LAYOUT[layout])
            now = [v.clone() for v in (y, h, gg, gx, gh)]
            first = first or now
            assert all(torch.equal(a, b) for a, b in zip(first, now))


@pytest.mark.parametrize("layout", ["tokens", "maps"])
def test_gradients_against_differences(layout):
    """<gradient, direction> against a central difference of the loss, both
    evaluated in 64 bits at the GPU's gradients.  The loss is smooth; with step
    1e-4 the difference's own error is about 1e-8 of its size, the gradients'
    about 1e-6 (n = 96 steps of 2^-24 and a few units each)."""
    N, T, C = 2, 96, 8
    d = inputs(20, N, T, C, "f32", layout, "logit")
    d["gate"] = d["gate"].clamp(-6, 6)
    y, h = torch.empty_like(d["x"]), torch.empty((N, C), device="cuda")
    st = bc.gated_scan_states(N, T, C, torch.float32, LAYOUT[layout])
    bc.gated_scan_fwd(d["gate"], d["x"], y, h0=d["h0"], h_last=h, states=st, layout=LAYOUT[layout])
    gg, gx, gh0 = torch.empty_like(y), torch.empty_like(y), torch.empty_like(h)
    bc.gated_scan_bwd(d["gate"], d["x"], st, d["gy"], gg, gx, grad_h_last=d["gh"], grad_h0=gh0, layout=LAYOUT[layout])
    s = lambda v: R.seq(to64(v), layout)
    gate, x, gy, h0, gh = s(d["gate"]), s(d["x"]), s(d["gy"]), to64(d["h0"]), to64(d["gh"])

    def loss(gate, x, h0):
        hs, yy, _ = R.scan_forward(gate, x, h0)
        return (yy * gy).sum() + (hs[T] * gh).sum()

    rng = np.random.default_rng(4)
    for name, at, grad in (("gate", gate, s(gg)), ("x", x, s(gx)), ("h0", h0, to64(gh0))):
        v, eps = rng.standard_normal(at.shape), 1e-4
        args = lambda sign: [(a + sign * eps * v) if n == name else a
                             for n, a in (("gate", gate), ("x", x), ("h0", h0))]
        diff = (loss(*args(1)) - loss(*args(-1))) / (2 * eps)
        dot, size = (grad * v).sum(), np.abs(grad * v).sum()
        assert abs(dot - diff) <= 1e-5 * size, (name, dot, diff)


@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,S", [(1, 1, 1), (3, 7, 9), (17, 65, 40), (130, 256, 130), (5, 1030, 5)])
def test_step(N, C, S, dt, form):
    say("scan step", N, C, S, dt, form)
    d = inputs(21, N, 1, C, dt, "tokens", form, packed=C % 8 == 0)
    gate, x = d["gate"][:, 0], d["x"][:, 0]
    pool = torch.randn((S, C), generator=torch.Generator().manual_seed(5)).cuda()
    perm = torch.randperm(S, generator=torch.Generator().manual_seed(6))[:N].to(torch.int32)
    cases = [(None, None)] if N > S else [(None, None), (perm.cuda(), None)]
    idle = perm.clone()
    idle[::2] = torch.tensor([-1, S, 2 ** 30, -2 ** 31], dtype=torch.int64).to(torch.int32).repeat(N)[:len(idle[::2])]
    cases += [(idle.cuda(), None), (perm.cuda(), "other")]
    for slots, where in cases:
        state = pool.clone()
        out = torch.full_like(pool, 7.0) if where else None
        y = torch.full((N, C), float("nan"), dtype=DT[dt], device="cuda")
        bc.gated_scan_step(gate, x, state, y, slots=slots, state_out=out, form=FORM[form])
        torch.cuda.synchronize()
        sl = np.arange(N) if slots is None else slots.cpu().numpy()
        on = (sl >= 0) & (sl < S)
        at = np.where(on, sl, 0)
        h, yy, e = R.scan_forward(to64(gate)[None], to64(x)[None], to64(pool)[at], None, form)
        close(y, np.where(on[:, None], yy[0], 0.0), e[1], dt, "y")
        new = out if where else state
        want = np.full((S, C), 7.0) if where else to64(pool)
        bound = np.zeros((S, C))
        want[sl[on]], bound[sl[on]] = h[1][on], e[1][on]
        close(new, want, bound, "f32", "state")
        if where:
            assert torch.equal(state, pool)


def test_step_continues_a_scan():
    """Prefill, then token by token: the states of one long scan."""
    N, T, C, cut = 3, 40, 64, 33
    d = inputs(22, N, T, C, "f32", "tokens", "logit")
    h = torch.empty((N, C), device="cuda")
    y = torch.empty((N, cut, C), device="cuda")
    bc.gated_scan_fwd(d["gate"][:, :cut], d["x"][:, :cut], y, h0=d["h0"], h_last=h)
    ys = [y]
    for t in range(cut, T):
        yt = torch.empty((N, C), device="cuda")
        bc.gated_scan_step(d["gate"][:, t], d["x"][:, t], h, yt)
        ys.append(yt[:, None])
    hh, yy, e = R.scan_forward(R.seq(to64(d["gate"]), "tokens"), R.seq(to64(d["x"]), "tokens"), to64(d["h0"]))
    close(torch.cat(ys, dim=1), R.unseq(yy, "tokens"), R.unseq(e[1:], "tokens"), "f32", "y")
    close(h, hh[T], e[T], "f32", "state")


def test_on_another_stream():
    N, T, C = 2, 300, 64
    d = inputs(23, N, T, C, "f32", "tokens", "logit")
    y0, y1 = torch.empty_like(d["x"]), torch.empty_like(d["x"])
    bc.gated_scan_fwd(d["gate"], d["x"], y0, h0=d["h0"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        bc.gated_scan_fwd(d["gate"], d["x"], y1, h0=d["h0"])
    s.synchronize()
    assert torch.equal(y0, y1)
