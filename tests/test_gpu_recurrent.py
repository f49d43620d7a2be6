"""The recurrent layer as a whole: training on a box layer's maps, serving in
8-bit codes, under HIP graphs, and at offsets past 32 bits."""
import sys

import numpy as np
import pytest
import torch

import oracle as O
from oracle import recurrent_oracle as R
from paper_1906_11367_amd import boxconv as bc
from paper_1906_11367_amd.layer import LayerPlan
from paper_1906_11367_amd.recurrent import RecurrentPlan, RecurrentServer

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("mix,bar", [("f32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("lengths", [None, [90, 0]])
def test_training_against_the_oracle(mix, bar, lengths):
    """Every output and gradient against 64 bits, normwise at the bars that the
    fp32 and the bf16 mix are held to (1e-4; operands rounded to 8 bits at up to
    four products in a row, 2^-8 each)."""
    N, C, T, D, M = 2, 24, 130, 16, 20
    plan = RecurrentPlan(N, C, T, D, M, mix_dtype=mix)
    x, gz = rand(1, N, C, T), rand(2, N, M, T)
    w_in, w_out = rand(3, 2 * D, C) / C ** 0.5, rand(4, M, D) / D ** 0.5
    h0, gh = rand(5, N, D), rand(6, N, D)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    dev = [v.cuda() for v in (x, w_in, w_out, gz, h0, gh)]
    z, h = plan.forward(dev[0], dev[1], dev[2], h0=dev[4], lengths=ln)
    dx, dwi, dwo, dh0 = plan.backward(dev[0], dev[1], dev[2], dev[3], grad_h_last=dev[5], lengths=ln)
    torch.cuda.synchronize()
    x, wi, wo, gz, h0, gh = (to64(v) for v in (x, w_in, w_out, gz, h0, gh))
    p = np.einsum("dc,nct->ndt", wi, x)
    s = lambda v: R.seq(v, "maps")
    gate, v = s(p[:, :D]), s(p[:, D:])
    hs, yy, _ = R.scan_forward(gate, v, h0, lengths)
    y = R.unseq(yy, "maps")
    dy = np.einsum("md,nmt->ndt", wo, gz)
    b = R.scan_backward(gate, v, s(dy), h0, gh, lengths)
    dp = np.concatenate([R.unseq(b["gate"], "maps"), R.unseq(b["x"], "maps")], axis=1)
    for name, got, want in (("z", z, np.einsum("md,ndt->nmt", wo, y)), ("h_last", h, hs[T]),
                            ("dx", dx, np.einsum("dc,ndt->nct", wi, dp)), ("dw_in", dwi, np.einsum("ndt,nct->dc", dp, x)),
                            ("dw_out", dwo, np.einsum("nmt,ndt->md", gz, y)), ("dh0", dh0, b["h0"])):
        err = np.linalg.norm(to64(got) - want) / np.linalg.norm(want)
        say(name, err)
        assert err <= bar, (name, err)


def test_on_a_box_layers_output():
    """The maps of a box layer scanned in raster order, as one network, forward
    and backward: the recurrent layer's input gradient feeds the box layer's."""
    N, C, H, W, B, M, D = 2, 8, 16, 12, 4, 24, 16
    box = LayerPlan(N, C, H, W, B, M, torch.float32, "f32")
    rec = RecurrentPlan(N, M, H * W, D, 10)
    x = rand(1, N, C, H, W).cuda()
    boxes = torch.cat([rand(2, C, B, 2), rand(3, C, B, 2).abs() + 0.5], dim=2).cuda()
    w = (rand(4, M, C * B) / 6).cuda()
    w_in, w_out = (rand(5, 2 * D, M) / 5).cuda(), (rand(6, 10, D) / 4).cuda()
    gz = rand(7, N, 10, H * W).cuda()
    maps = box.forward(x, boxes, w).view(N, M, H * W)
    rec.forward(maps, w_in, w_out)
    dmaps = rec.backward(maps, w_in, w_out, gz)[0]
    dx, dboxes, dw = box.backward(x, boxes, w, dmaps.view(N, M, H, W))
    torch.cuda.synchronize()
    # the loss as a function of the first 1x1 weights, by a difference in 64 bits
    o = O.box_forward(x.cpu().numpy(), boxes.cpu().numpy()).reshape(N, C * B, H * W).astype(np.float64)
    wi, wo, g, w0 = to64(w_in), to64(w_out), to64(gz), to64(w)

    def loss(w1):
        p = np.einsum("dm,nmt->ndt", wi, np.einsum("mk,nkt->nmt", w1, o))
        _, yy, _ = R.scan_forward(R.seq(p[:, :D], "maps"), R.seq(p[:, D:], "maps"))
        return (np.einsum("md,ndt->nmt", wo, R.unseq(yy, "maps")) * g).sum()

    v = np.random.default_rng(1).standard_normal(w0.shape)
    diff, dot = (loss(w0 + 1e-5 * v) - loss(w0 - 1e-5 * v)) / 2e-5, (to64(dw) * v).sum()
    assert abs(diff - dot) <= 1e-4 * np.abs(to64(dw) * v).sum()
    assert torch.isfinite(dx).all() and torch.isfinite(dboxes).all()


def make_server(D, C, M, S, seed=1):
    w_in, w_out = (rand(seed, 2 * D, C) / C ** 0.5).cuda(), (rand(seed + 1, M, D) / D ** 0.5).cuda()
    b_in, b_out = rand(seed + 2, 2 * D).cuda(), rand(seed + 3, M).cuda()
    return RecurrentServer(w_in, w_out, S, b_in=b_in, b_out=b_out)


def expect(server, x, h0, T):
    """z and the last state of tokens x [N, T, C] in 64 bits, every intermediate
    rounded as the server stores it (bf16)."""
    N = x.shape[0]
    bf = lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16).float().numpy().astype(np.float64)
    qi, si = (v.cpu().numpy() for v in server.w_in)
    qo, so = (v.cpu().numpy() for v in server.w_out)
    D, C = server.D, server.C
    q, s = R.codes(x.reshape(-1, C))
    p = bf(R.mix_codes(q, s, qi[:, :C], si, to64(server.b_in))[0]).reshape(N, T, 2 * D)
    h, yy, _ = R.scan_forward(R.seq(p[..., :D], "tokens"), R.seq(p[..., D:], "tokens"), h0)
    q, s = R.codes(bf(R.unseq(yy, "tokens")).reshape(-1, D))
    z = R.mix_codes(q, s, qo[:, :D], so, to64(server.b_out))[0].reshape(N, T, server.M)
    return z, h[T]


def near(got, want, what):
    """A value of the chain may round to the neighbouring bf16 or code in 64 bits
    where it lies between two: such a flip moves z by one part in 127 of a term
    or so.  Normwise 2e-3 beside the 2^-9 of the outputs' own rounding."""
    err = np.linalg.norm(to64(got) - want) / np.linalg.norm(want)
    say(what, err)
    assert err <= 2e-3 + 2.0 ** -9, (what, err)


@pytest.mark.parametrize("layout", [bc.BC_TOKENS, bc.BC_MAPS])
def test_serving(layout):
    """Prompts, then tokens one at a time, in slots of a pool; idle rows."""
    D, C, M, S, N, T = 64, 48, 40, 9, 3, 37
    server = make_server(D, C, M, S)
    x = rand(9, N, T + 3, C).to(torch.bfloat16).cuda()
    slots = torch.tensor([7, 0, 4], dtype=torch.int32, device="cuda")
    prompt = x[:, :T].contiguous()
    given = prompt if layout == bc.BC_TOKENS else prompt.transpose(1, 2).contiguous()
    z = server.prefill(given, slots, layout=layout)
    want, h = expect(server, to64(prompt).astype(np.float32), np.zeros((N, D)), T)
    near(z if layout == bc.BC_TOKENS else z.transpose(1, 2), want, "prefill")
    near(server.state[slots.long()], h, "state")
    for t in range(T, T + 3):
        before = to64(server.state)
        rows = torch.tensor([7, -1, 4], dtype=torch.int32, device="cuda") if t == T + 1 else slots
        z = server.step(x[:, t], rows)
        want, h = expect(server, to64(x[:, t:t + 1]).astype(np.float32), before[slots.cpu().numpy()], 1)
        live = rows.cpu().numpy() >= 0
        near(z[torch.from_numpy(live)], want[live, 0], "step")
        near(server.state[slots.long()[torch.from_numpy(live).cuda()]], h[live], "state")
        others = [s for s in range(S) if s not in rows.tolist()]
        assert np.array_equal(to64(server.state)[others], before[others])


def test_prompt_in_two_parts():
    D, C, M, N, T, cut = 32, 40, 24, 2, 300, 140
    one, two = make_server(D, C, M, 4), make_server(D, C, M, 4)
    x = rand(3, N, T, C).to(torch.bfloat16).cuda()
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    z = one.prefill(x, slots)
    a = two.prefill(x[:, :cut], slots)
    b = two.prefill(x[:, cut:], slots, fresh=False)
    near(torch.cat([a, b], dim=1), to64(z), "z")
    near(two.state, to64(one.state), "state")


def test_under_graphs():
    """A decoding step and a training step captured into HIP graphs: replays,
    with eager work between them, give the eager results bit for bit."""
    server = make_server(64, 256, 128, 40)
    x, slots = rand(1, 40, 256).to(torch.bfloat16).cuda(), torch.arange(40, dtype=torch.int32, device="cuda")
    N, T, C = 2, 700, 64
    gate, v, gy = (rand(s, N, T, C).cuda() for s in (2, 3, 4))
    y, gg, gx = (torch.empty_like(gate) for _ in range(3))
    st = bc.gated_scan_states(N, T, C)
    ws = torch.empty(max(bc.gated_scan_workspace_bytes(op, N, T, C, bc.BC_F32) for op in (0, 1)), dtype=torch.uint8,
                     device="cuda")
    mx = rand(5, 1, 512, 300).cuda()
    wq, wsc = server._codes(rand(6, 96, 512).cuda())
    mz = torch.empty((1, 96, 300), device="cuda")

    def work():
        z = server.step(x, slots)
        bc.gated_scan_fwd(gate, v, y, states=st, ws=ws)
        bc.gated_scan_bwd(gate, v, st, gy, gg, gx, ws=ws)
        bc.pointwise_mix_i8(wq, wsc, mx, mz, layout=bc.BC_MAPS)
        return z

    def fresh():
        server.state.copy_(start)
        for o in (y, gg, gx, mz):
            o.fill_(float("nan"))

    start = rand(7, 40, 64).cuda()
    fresh()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        eager = [t.clone() for t in (work(), y, gg, gx, mz, server.state)]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = work()
    for i in range(3):
        fresh()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, a, b in zip("z y gg gx mz state".split(), (z, y, gg, gx, mz, server.state), eager):
            assert torch.equal(a, b), (i, name)
        (gate @ gate.transpose(1, 2).contiguous()).sum()   # eager work in between


def test_offsets_past_32_bits_scan():
    """2.2 billion elements: the last steps of the last sequence, which a reset
    cuts off from the rest, in both layouts."""
    N, C, tail = 2, 1024, 150
    T = (2 ** 31 + 2 ** 27) // (N * C)
    for layout in ("tokens", "maps"):
        say("large", layout)
        shape = (N, T, C) if layout == "tokens" else (N, C, T)
        gate, x = (torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2))
        last = (lambda v: v[-1, T - tail:]) if layout == "tokens" else (lambda v: v[-1, :, T - tail:].t())
        last(gate)[0] = -float("inf")
        y = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        code = bc.BC_TOKENS if layout == "tokens" else bc.BC_MAPS
        st = bc.gated_scan_states(N, T, C, torch.bfloat16, code)
        h = torch.empty((N, C), device="cuda")
        bc.gated_scan_fwd(gate, x, y, h_last=h, states=st, layout=code)
        g, v = (to64(last(t))[:, None, :] for t in (gate, x))
        hs, yy, e = R.scan_forward(g, v)
        assert (np.abs(to64(last(y))[:, None] - yy) <= e[1:] + R.U_BF16 * np.abs(yy)).all()
        assert (np.abs(to64(h[-1])[None] - hs[tail]) <= e[tail] + R.EPS * np.abs(hs[tail])).all()
        del y
        gy = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_()
        gg, gx = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        bc.gated_scan_bwd(gate, x, st, gy, gg, gx, layout=code)
        b = R.scan_backward(g, v, to64(last(gy))[:, None, :])
        for name, got in (("gate", gg), ("x", gx)):
            want, bound = b[name][1:], b[name + "_bound"][1:]   # the reset's own gradient needs the state before
            err = np.abs(to64(last(got))[1:, None] - want)
            assert (err <= bound + R.U_BF16 * (np.abs(want) + bound)).all(), name
        del gate, x, gy, gg, gx, st
        torch.cuda.empty_cache()


def test_offsets_past_32_bits_mix_and_step():
    K, M, T = 8192, 72, (2 ** 31 + 2 ** 26) // 8192
    say("large mix")
    wq, ws = RecurrentServer._codes(rand(1, M, K).cuda())
    x = torch.empty((T, K), dtype=torch.bfloat16, device="cuda").normal_()
    out = torch.empty((T, M), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, out)
    z, b = R.mix_codes(*R.codes(to64(x[-40:]).astype(np.float32)), wq.cpu().numpy(), ws.cpu().numpy())
    assert (np.abs(to64(out[-40:]) - z) <= b + R.EPS * np.abs(z)).all()
    del x, out
    torch.cuda.empty_cache()
    N, K, P = 2, 1024, 2 ** 20 + 2 ** 16 + 40
    say("large maps")
    wq, ws = RecurrentServer._codes(rand(2, 8, K).cuda())
    x = torch.empty((N, K, P), dtype=torch.bfloat16, device="cuda").normal_()
    out = torch.empty((N, 8, P), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, out, layout=bc.BC_MAPS)
    z, b = R.mix_codes(*R.codes(to64(x[-1, :, -70:]).T.astype(np.float32)), wq.cpu().numpy(), ws.cpu().numpy())
    assert (np.abs(to64(out[-1, :, -70:]).T - z) <= b + R.EPS * np.abs(z)).all()
    del x, out
    torch.cuda.empty_cache()
    say("large pool")
    S, C = 2 ** 19 + 2 ** 15, 4096
    pool = torch.zeros((S, C), device="cuda")
    slots = torch.tensor([S - 1, 3, S - 2], dtype=torch.int32, device="cuda")
    gate, v = rand(3, 3, C).cuda(), rand(4, 3, C).cuda()
    h = rand(5, 3, C).cuda()
    pool[slots.long()] = h
    y = torch.empty((3, C), device="cuda")
    bc.gated_scan_step(gate, v, pool, y, slots=slots)
    hs, yy, e = R.scan_forward(to64(gate)[None], to64(v)[None], to64(h))
    assert (np.abs(to64(y) - yy[0]) <= e[1] + R.EPS * np.abs(yy[0])).all()
    assert torch.equal(pool[slots.long()], y)
