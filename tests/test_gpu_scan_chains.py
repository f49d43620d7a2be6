"""Chained tiles of the gated scan across the groups of their look-back (16 tiles of
128 steps, 2048 steps), in the cut that most long calls take: against 64 bits,
at lengths around a group's edges, under aliases and beside another call."""
import sys

import numpy as np
import pytest
import torch

from oracle import recurrent_oracle as R
from paper_1906_11367_amd import boxconv as bc
from test_gpu_scan import close, inputs, run_both, to64

pytestmark = pytest.mark.gpu

# one whole group; a last group of one tile, of which one step; three groups
SIZES = [(2, 2048, 70, None), (2, 2049, 130, None), (3, 4200, 200, None), (1, 6145, 40, None),
         (3, 2049, 66, [2047, 2048, 2049]), (4, 4200, 70, [4096, 4097, 0, 4200]), (3, 4224, 64, [1, 2176, 4095])]


@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,C,lengths", SIZES)
def test_groups(N, T, C, lengths, dt, form):
    print("scan groups", N, T, C, lengths, dt, form, flush=True)
    sys.stdout.flush()
    d = inputs(31, N, T, C, dt, "tokens", form)
    if lengths is not None:
        dead = (torch.arange(T)[None, :] >= torch.tensor(lengths)[:, None])[:, :, None].cuda()
        d.update({k: d[k].masked_fill(dead, float("nan")) for k in ("gate", "x", "gy")})
    run_both(d, N, T, C, dt, "tokens", form, lengths)


def test_groups_of_long_memories():
    """Coefficients near 1, so that a state of the first tile still counts in the
    last: the carries alone make the difference between the groups."""
    N, T, C = 2, 4200, 72
    d = inputs(32, N, T, C, "f32", "tokens", "value")
    d["gate"] = 1.0 - d["gate"].abs() * 2.0 ** -11
    d["x"] = d["x"] * 2.0 ** -6
    assert (d["gate"].double().prod(dim=1) > 0.05).all()
    run_both(d, N, T, C, "f32", "tokens", "value")


def test_bf16_outputs_of_fp32_inputs():
    N, T, C = 2, 2200, 72
    run_both(inputs(33, N, T, C, "f32", "tokens", "logit", packed=True), N, T, C, "f32", "tokens", "logit", out_dt="bf16",
             packed_grad=True)


@pytest.mark.parametrize("layout", ["tokens", "maps"])
@pytest.mark.parametrize("T", [1, 5, 100, 600, 2500])
def test_states_and_their_gradients_in_place(T, layout):
    """h_last = h0 and grad_h0 = grad_h_last: the same bits as apart."""
    N, C = 2, 48
    code = bc.BC_TOKENS if layout == "tokens" else bc.BC_MAPS
    d = inputs(34, N, T, C, "bf16", layout, "logit")
    new = lambda: torch.full_like(d["x"], float("nan"))
    results = []
    for alias in (False, True):
        y, gg, gx = new(), new(), new()
        h0, gh = d["h0"].clone(), d["gh"].clone()
        h, gh0 = (h0, gh) if alias else (torch.empty_like(h0), torch.empty_like(gh))
        st = bc.gated_scan_states(N, T, C, torch.bfloat16, code)
        bc.gated_scan_fwd(d["gate"], d["x"], y, h0=h0, h_last=h, states=st, layout=code)
        bc.gated_scan_bwd(d["gate"], d["x"], st, d["gy"], gg, gx, grad_h_last=gh, grad_h0=gh0, layout=code)
        results.append((y, h, gg, gx, gh0))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    _, _, e = R.scan_forward(R.seq(to64(d["gate"]), layout), R.seq(to64(d["x"]), layout), to64(d["h0"]))
    h, _, _ = R.scan_forward(R.seq(to64(d["gate"]), layout), R.seq(to64(d["x"]), layout), to64(d["h0"]))
    close(results[1][1], h[T], e[T], "f32", "h_last")


def test_two_chained_scans_at_once():
    """On two streams, each with a workspace of its own, blocks of both on the chip
    together: the bits of each alone."""
    sizes = [(8, 6000, 512), (2, 9000, 1024)]
    work = []
    for i, (N, T, C) in enumerate(sizes):
        g = torch.Generator(device="cuda").manual_seed(i)
        gate, x, gy = (torch.randn((N, T, C), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
        ws = [torch.empty(bc.gated_scan_workspace_bytes(op, N, T, C, bc.BC_BF16), dtype=torch.uint8, device="cuda")
              for op in (0, 1)]
        work.append((gate, x, gy, bc.gated_scan_states(N, T, C, torch.bfloat16), ws,
                     [torch.empty_like(x) for _ in range(3)]))

    def both(gate, x, gy, st, ws, out):
        bc.gated_scan_fwd(gate, x, out[0], states=st, ws=ws[0])
        bc.gated_scan_bwd(gate, x, st, gy, out[1], out[2], ws=ws[1])

    want = []
    for w in work:
        both(*w)
        torch.cuda.synchronize()
        want.append([o.clone() for o in w[-1]])
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    for _ in range(4):
        for w, s in zip(work, streams):
            with torch.cuda.stream(s):
                for o in w[-1]:
                    o.fill_(7.0)
                both(*w)
        torch.cuda.synchronize()
        for w, refs in zip(work, want):
            for o, ref in zip(w[-1], refs):
                assert torch.equal(o, ref)


@pytest.mark.parametrize("layout", ["tokens", "maps"])
@pytest.mark.parametrize("T", [133, 2100])
def test_wide_strides_bf16(layout, T):
    """Rows and batches an odd number of elements apart, NaN between them."""
    N, C = 2, 41
    d = inputs(35, N, T, C, "bf16", layout, "logit")
    for k in ("gate", "x"):
        n, r, c = d[k].shape
        big = torch.full((N + 1, r + 2, c + 3 + c % 2), float("nan"), dtype=torch.bfloat16, device="cuda")
        view = big[:N, :r, :c]
        view.copy_(d[k])
        d[k] = view
    run_both(d, N, T, C, "bf16", layout, "logit")
