"""A linear-attention block as a whole: training against 64 bits and differences,
serving in 8-bit codes, under a graph."""
import sys

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_1906_11367_amd import boxconv as bc
from paper_1906_11367_amd.attention import LinearAttentionPlan, LinearAttentionServer

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def weights(plan_shape, C, H, Dv, seed=1):
    W, E = plan_shape.width, H * Dv
    w = {"w_pre": 1 + 0.2 * rand(seed, C), "w_in": rand(seed + 1, C, W) / C ** 0.5, "w_head": 1 + 0.2 * rand(seed + 2, E),
         "w_out": rand(seed + 3, E, C) / E ** 0.5, "w_post": 1 + 0.2 * rand(seed + 4, C), "res_scale": 0.5 + 0.1 * rand(seed + 5, C)}
    at, n = plan_shape.columns[4]
    w["w_in"][:, at:at + n] += 0.3   # (memories of a few tokens and more)
    return {k: v.cuda() for k, v in w.items()}


def exactly(v):
    return v


def to_bf16(v):
    return torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16).double().numpy()


def block(x, w, shape, eps, s0=None, lengths=None, lo=exactly, lo_w=exactly):
    """The block in 64 bits: r, s_last and what the backward needs.  lo, lo_w: round
    what the plan stores, and what its products take of the matrices."""
    N, T, C = x.shape
    flat = lambda v: v.reshape(N * T, -1)
    xn = lo(A.block_norm(flat(x), w_pre=w["w_pre"], eps=eps)["y"][0])
    p = lo(xn @ lo_w(w["w_in"])).reshape(N, T, -1)
    cut = [p[..., at:at + n] for at, n in shape.columns]
    heads = ((shape.H, shape.Dk), (shape.Hk, shape.Dk), (shape.Hk, shape.Dv))
    q, k, v = (c.reshape(N, T, *h) for c, h in zip(cut, heads))
    gate, logits = cut[3], cut[4]
    at = A.attention(q, k, v, logits, "logit", shape.scale, s0, lengths)
    o = lo(flat(at["y"][0]))
    m = lo(A.block_norm(o, gate=flat(gate), w_post=w["w_head"], groups=shape.H, eps=eps, pre=False)["r"][0])
    z = lo(m @ lo_w(w["w_out"]))
    r = A.block_norm(z, x=flat(x), w_post=w["w_post"], res_scale=w["res_scale"], groups=1, eps=eps, pre=False)["r"][0]
    return r.reshape(N, T, C), at["s_last"][0], (xn, q, k, v, gate, logits, o, m, z)


def block_grads(x, w, shape, eps, kept, dr, s0, ds, lengths, lo=exactly, lo_w=exactly):
    N, T, C = x.shape
    flat = lambda v: v.reshape(N * T, -1)
    xn, q, k, v, gate, logits, o, m, z = kept
    n3 = A.block_norm(z, x=flat(x), w_post=w["w_post"], res_scale=w["res_scale"], groups=1, eps=eps, pre=False, dr=flat(dr))
    dz, dres = lo(n3["dz"][0]), lo(n3["dx"][0])
    dm = lo(dz @ lo_w(w["w_out"]).T)
    n2 = A.block_norm(o, gate=flat(gate), w_post=w["w_head"], groups=shape.H, eps=eps, pre=False, dr=dm)
    g = A.attention(q, k, v, logits, "logit", shape.scale, s0, lengths, lo(n2["dz"][0]).reshape(N, T, shape.H, shape.Dv), ds)
    dp = np.zeros((N, T, shape.width))
    for (at, n), d in zip(shape.columns, (g["dq"][0], g["dk"][0], g["dv"][0], n2["dgate"][0], g["dgate"][0])):
        dp[..., at:at + n] = d.reshape(N, T, n)
    dp = lo(flat(dp))
    n1 = A.block_norm(flat(x), w_pre=w["w_pre"], eps=eps, dr=dres, dy=lo(dp @ lo_w(w["w_in"]).T))
    return {"dx": n1["dz"][0].reshape(N, T, C), "ds0": g["ds0"][0], "w_pre": n1["dw_pre"][0], "w_in": xn.T @ dp,
            "w_head": n2["dw_post"][0], "w_out": m.T @ dz, "w_post": n3["dw_post"][0], "res_scale": n3["dres_scale"][0]}


# fp32: two products, the attention and three norms each way, at 1e-4 the bar that
# the fp32 mix is held to.  bf16: the oracle rounds where the plan stores.  A norm
# divides by its row's size, so the gradients of rows that come out small follow
# their roundings far: at these inputs the roundings alone, in 64 bits, move dx and
# w_in's gradient by 12 and 15 % where keys are shared, and by 3 % where not.  What is
# left between plan and oracle are values that round to the other side: the attention's
# sums are off by 2^-17 rms of themselves, so one in 2^-17 / 2^-8 of its values steps by
# 2^-7, sqrt(12) times a rounding's rms of 2^-7 / sqrt(12).  Squares add up:
# sqrt(2^-9 * 12) = 15 % of what all roundings do, 2.3e-2 at most; the bar is 4e-2.
@pytest.mark.parametrize("dtype,bar", [("f32", 1e-4), ("bf16", 4e-2)])
@pytest.mark.parametrize("Hk,lengths", [(None, None), (2, [150, 37])])
def test_training_against_the_oracle(dtype, bar, Hk, lengths):
    N, T, C, H, Dk, Dv = 2, 150, 40, 4, 16, 24
    plan = LinearAttentionPlan(N, T, C, H, Dk, Dv, Hk=Hk, dtype=dtype)
    w = weights(plan.shape, C, H, Dv)
    t = plan.t
    x, dr = rand(10, N, T, C).to(t).cuda(), rand(11, N, T, C).to(t).cuda()
    s0, ds = rand(12, N, H, Dk, Dv).cuda(), rand(13, N, H, Dk, Dv).cuda()
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    r, s_last = plan.forward(x, w, s0=s0, lengths=ln)
    dx, grads, ds0 = plan.backward(x, w, dr, grad_s_last=ds, lengths=ln)
    torch.cuda.synchronize()
    w64 = {k: to64(v) for k, v in w.items()}
    lo = (to_bf16,) * 2 if dtype == "bf16" else (exactly,) * 2
    wr, ws, kept = block(to64(x), w64, plan.shape, plan.eps, to64(s0), lengths, *lo)
    want = block_grads(to64(x), w64, plan.shape, plan.eps, kept, to64(dr), to64(s0), to64(ds), lengths, *lo)
    got = {"dx": dx, "ds0": ds0, **grads}
    for name, a, b in [("r", r, wr), ("s_last", s_last, ws)] + [(n, got[n], want[n]) for n in got]:
        err = np.linalg.norm(to64(a) - b) / np.linalg.norm(b)
        say(name, err)
        assert err <= bar, (name, err)


def test_training_of_odd_sizes():
    """No size a whole vector, a few tokens, an empty sequence; fp32 and its bar."""
    N, T, C, H, Dk, Dv = 3, 5, 33, 3, 7, 5
    plan = LinearAttentionPlan(N, T, C, H, Dk, Dv, Hk=1)
    w = weights(plan.shape, C, H, Dv)
    x, dr = rand(14, N, T, C).cuda(), rand(15, N, T, C).cuda()
    lengths = [5, 0, 4]
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    r, s_last = plan.forward(x, w, lengths=ln)
    dx, grads, ds0 = plan.backward(x, w, dr, lengths=ln)
    torch.cuda.synchronize()
    w64, none = {k: to64(v) for k, v in w.items()}, np.zeros((N, H, Dk, Dv))
    wr, ws, kept = block(to64(x), w64, plan.shape, plan.eps, none, lengths)
    want = block_grads(to64(x), w64, plan.shape, plan.eps, kept, to64(dr), none, none, lengths)
    got = {"dx": dx, "ds0": ds0, **grads}
    for name, a, b in [("r", r, wr), ("s_last", s_last, ws)] + [(n, got[n], want[n]) for n in got]:
        err = np.linalg.norm(to64(a) - b) / np.linalg.norm(b)
        say(name, err)
        assert err <= 1e-4, (name, err)
    assert torch.equal(r[1], x[1]) and (s_last[1] == 0).all()


def test_the_oracles_gradients_are_the_losss_differences():
    """Along a random direction of every weight and of x, in 64 bits."""
    N, T, C, H, Dk, Dv = 1, 9, 6, 2, 3, 4
    shape = LinearAttentionPlan(N, T, C, H, Dk, Dv).shape
    w = {k: to64(v) for k, v in weights(shape, C, H, Dv).items()}
    x, dr, ds, s0 = (to64(rand(20 + i, *s)) for i, s in enumerate(((N, T, C), (N, T, C), (N, H, Dk, Dv), (N, H, Dk, Dv))))

    def loss(x, w):
        r, s, _ = block(x, w, shape, 1e-6, s0)
        return (r * dr).sum() + (s * ds).sum()

    _, _, kept = block(x, w, shape, 1e-6, s0)
    g = block_grads(x, w, shape, 1e-6, kept, dr, s0, ds, None)
    rng = np.random.default_rng(1)
    for name in ["dx"] + list(w):
        at = x if name == "dx" else w[name]
        v, e = rng.standard_normal(at.shape), 1e-6
        f = lambda s: loss(x + s * v, w) if name == "dx" else loss(x, {**w, name: at + s * v})
        dot = (g[name] * v).sum()
        assert abs((f(e) - f(-e)) / (2 * e) - dot) <= 1e-6 * (1 + np.abs(g[name] * v).sum()), name


def make_server(C=64, H=4, Dk=16, Dv=32, Hk=2, slots=6):
    shape = LinearAttentionPlan(1, 1, C, H, Dk, Dv, Hk=Hk, with_backward=False).shape
    w = weights(shape, C, H, Dv)
    return LinearAttentionServer(w, H, Dk, Dv, slots, Hk=Hk), w, shape


def decoded(codes, K):
    q, s = codes
    return to64(q)[:, :K].T * to64(s)[None, :]


# Activations are taken in codes of step m / 127, m a row's largest value: for rows
# of about 64 to 128 values of one spread m is below 4 of them, so a code is off by
# at most 1.6 % and by 0.9 % rms; two products, and six roundings of 2^-8: 2 * 0.9 % +
# sqrt(6) 0.23 % < 3 % of what the block adds, which norms and the gate pass on.
BAR = 5e-2


def test_serving_against_the_oracle():
    """Ragged prompts with an idle row, then tokens, against 64 bits on the decoded
    weights."""
    server, w, shape = make_server()
    C, N, T = server.C, 4, 40
    w64 = {k: to64(v) for k, v in w.items()}
    w64["w_in"], w64["w_out"] = decoded(server.w_in, C), decoded(server.w_out, shape.H * shape.Dv)
    x = rand(30, N, T + 3, C).to(torch.bfloat16).cuda()
    slots = torch.tensor([5, -1, 0, 2], dtype=torch.int32, device="cuda")
    lengths = [40, 40, 17, 33]
    r = server.prefill(x[:, :T].contiguous(), slots, torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    state = np.zeros((N, shape.H, shape.Dk, shape.Dv))
    live = [0, 2, 3]
    for n in live:
        wr, state[n:n + 1], _ = block(to64(x[n:n + 1, :lengths[n]]), w64, shape, server.eps, lo=to_bf16)
        add, want = to64(r[n, :lengths[n]]) - to64(x[n, :lengths[n]]), wr[0] - to64(x[n, :lengths[n]])
        err = np.linalg.norm(add - want) / np.linalg.norm(want)
        say("prompt", n, err)
        assert err <= BAR
        got = to64(server.state[int(slots[n])])
        assert np.linalg.norm(got - state[n]) <= BAR * np.linalg.norm(state[n])
    assert (server.state[[1, 3, 4]] == 0).all()
    for t in range(T, T + 3):
        xt = x[:, t].contiguous()
        r = server.step(xt, slots)
        for n in live:
            wr, state[n:n + 1], _ = block(to64(xt[n:n + 1])[:, None], w64, shape, server.eps, state[n:n + 1], lo=to_bf16)
            add, want = to64(r[n]) - to64(xt[n]), wr[0, 0] - to64(xt[n])
            err = np.linalg.norm(add - want) / np.linalg.norm(want)
            say("token", t, n, err)
            assert err <= BAR
        assert torch.equal(r[1], xt[1])   # the idle row
    assert (server.state[[1, 3, 4]] == 0).all()


def test_a_prompt_in_two_parts():
    """The second part from the pool's states: what one prompt gives."""
    server, _, _ = make_server()
    x = rand(31, 2, 60, server.C).to(torch.bfloat16).cuda()
    slots = torch.tensor([1, 4], dtype=torch.int32, device="cuda")
    whole = server.prefill(x, slots)
    state = server.state.clone()
    server.state = torch.zeros_like(state)
    a = server.prefill(x[:, :25].contiguous(), slots)
    b = server.prefill(x[:, 25:].contiguous(), slots, fresh=False)
    # the same tokens' codes; the attention's chunks lie otherwise, so a value now
    # and then rounds to the next bf16 and moves its row's codes by one
    err = (torch.cat([a, b], 1).float() - whole.float()).norm() / whole.float().norm()
    assert err <= 2.0 ** -8 and (server.state - state).norm() <= 2.0 ** -8 * state.norm()


def test_under_a_graph():
    """A training step and a serving step, captured once and replayed on other
    inputs, with eager work between."""
    N, T, C, H, Dk, Dv = 2, 70, 32, 2, 16, 16
    plan = LinearAttentionPlan(N, T, C, H, Dk, Dv, dtype="bf16")
    w = weights(plan.shape, C, H, Dv)
    server = LinearAttentionServer(w, H, Dk, Dv, 4)
    x, dr = torch.zeros((2, N, T, C), dtype=torch.bfloat16, device="cuda")
    token, slots = torch.zeros((3, C), dtype=torch.bfloat16, device="cuda"), torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda")

    def step():
        r, s = plan.forward(x, w)
        dx, g, _ = plan.backward(x, w, dr)
        return [r, s, dx, *g.values(), server.step(token, slots)]

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for seed in (40, 50, 60):
        x.copy_(rand(seed, N, T, C))
        dr.copy_(rand(seed + 1, N, T, C))
        token.copy_(rand(seed + 2, 3, C))
        server.state.fill_(0.5)
        want = [t.clone() for t in step()] + [server.state.clone()]
        server.state.fill_(0.5)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out + [server.state], want):
            assert torch.equal(a, b)


def test_refusals():
    with pytest.raises(ValueError):
        LinearAttentionPlan(1, 8, 8, 4, 8, 8, Hk=3)
    with pytest.raises(ValueError):
        LinearAttentionPlan(1, 8, 8, 4, 8, 8, dtype="f16")
    with pytest.raises(ValueError):
        LinearAttentionPlan(2, 65536, 8, 4, 8, 8)
    server, w, shape = make_server()
    with pytest.raises(ValueError):
        LinearAttentionServer({**w, "w_in": w["w_in"][:, :-8]}, shape.H, shape.Dk, shape.Dv, 4, Hk=shape.Hk)
    with pytest.raises(bc.BoxConvError):
        server.step(rand(1, 2, server.C).cuda())
    with pytest.raises(bc.BoxConvError):
        server.prefill(rand(1, 2, 3, server.C).to(torch.bfloat16).cuda(), torch.tensor([0.0, 1.0], device="cuda"))
