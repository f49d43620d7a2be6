"""The operators of a recurrent layer as its users call them, as measurable cases.

A recurrent layer mixes along a sequence with a gated linear recurrence, one
state per channel, and across channels with matrix products.  Three calls carry
it: the gated scan over whole sequences (forward, and with its backward), the
scan's step for one new token of every running sequence, and the 1x1 mix in
8-bit integers, with a scale for each token and each output channel.

  kind    "scan"  the forward over whole sequences: outputs and last states
          "train" the forward and the backward: every gradient as well
          "step"  one token for N sequences whose states live in a pool
          "mix"   tokens [T, K] by weights [M, K]
          "maps"  maps [N, K, P] by weights [M, K], giving maps [N, M, P]
  dt      "bf16" or "f32": the type of the tensors that go in and come out
          (the mixes' outputs have their own, out)
  layout  "tokens" [N, T, C] (channels contiguous) or "maps" [N, C, T] (time
          contiguous, as the 1x1 mix writes its maps)
  form    "logit": a = sigmoid(gate), h_t = a_t h_{t-1} + (1 - a_t) x_t
          "value": a = gate itself,   h_t = a_t h_{t-1} + x_t
  ragged  every sequence has its own length (one of them zero, one full);
          outputs and gradients past it are zero, the last state is that at it
  packed  gate and x are the two halves of one projection's output
  start   an initial state is given (zero otherwise), and its gradient asked for
  bias, relu  the mix's epilogue

The integer codes of the mix, for each token's K values x (and once, ahead of
time, for each weight row): with m = max |x|, in 32-bit arithmetic,
  scale = m / 127,  q = round to nearest even(x * (127 / m))
(all zero where m < 2^-100); the product of the codes is exact, and the output
is product * scale of the token * scale of the weight row + bias.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_TINY = 2.0 ** -100


def _scan(name, kind, N, T, C, dt, layout="tokens", form="logit", ragged=False, packed=True, start=False):
    return {"name": name, "kind": kind, "N": N, "T": T, "C": C, "dt": dt, "layout": layout, "form": form,
            "ragged": ragged, "packed": packed, "start": start}


def _mix(name, T, K, M, dt, out, bias=False, relu=False):
    return {"name": name, "kind": "mix", "T": T, "K": K, "M": M, "dt": dt, "out": out, "bias": bias, "relu": relu}


def listed():
    return [
        # one new token for a handful of sequences: latency only
        {"name": "step_8", "kind": "step", "N": 8, "C": 1024, "S": 8, "dt": "bf16", "form": "logit"},
        # a full serving batch, its states scattered in a pool, a few rows idle
        {"name": "step_512", "kind": "step", "N": 512, "C": 4096, "S": 1024, "dt": "bf16", "form": "logit"},
        # a batch of short prompts
        _scan("scan_short", "scan", 16, 128, 1024, "bf16"),
        # one long document: few rows, all the work along the time axis
        _scan("scan_long", "scan", 1, 65536, 1024, "bf16", start=True),
        # the layer in training on token sequences
        _scan("train_tokens", "train", 8, 4096, 2048, "bf16"),
        # odd sizes, padded sequences, coefficients given as they are
        _scan("train_ragged", "train", 6, 1531, 837, "f32", form="value", ragged=True, packed=False, start=True),
        # the layer in training on the maps of square crops (64 x 64), as the fp32 mix writes them
        _scan("train_maps", "train", 32, 64 * 64, 256, "f32", layout="maps"),
        # one token through a wide projection: the weights are all there is to read
        _mix("mix_1", 1, 4096, 8192, "bf16", "bf16"),
        # a decoding batch
        _mix("mix_24", 24, 2048, 8192, "bf16", "bf16", bias=True),
        # odd sizes everywhere, fp32 in and out
        _mix("mix_odd", 777, 1000, 1537, "f32", "f32", bias=True, relu=True),
        # a large prefill batch: bound by the matrix units
        _mix("mix_large", 16384, 4096, 8192, "bf16", "bf16"),
        # the 1x1 mix after the boxes on a batch of square crops, deployed
        {"name": "maps_pose", "kind": "maps", "N": 32, "K": 1024, "P": 64 * 64, "M": 256, "dt": "bf16",
         "out": "f32", "bias": False, "relu": True},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scan", "train", "step", "mix", "mix", "maps"])
    dt = rng.choice(["bf16", "f32"])
    if kind == "step":
        N = _logint(rng, 1, 512)
        return {"kind": kind, "N": N, "C": _logint(rng, 64, 4096), "S": N + _logint(rng, 1, 512), "dt": dt,
                "form": rng.choice(["logit", "value"])}
    if kind in ("scan", "train"):
        while True:
            N, T, C = _logint(rng, 1, 256), _logint(rng, 1, 65536), _logint(rng, 24, 4096)
            if 2 ** 14 <= N * T * C <= 2 ** 26:
                break
        packed = rng.random() < 0.5
        if packed:   # halves of one projection: whole vectors of 16 bytes
            C = (C + 7) // 8 * 8
        return {"kind": kind, "N": N, "T": T, "C": C, "dt": dt, "layout": rng.choice(["tokens", "tokens", "maps"]),
                "form": rng.choice(["logit", "value"]), "ragged": rng.random() < 0.4, "packed": packed,
                "start": rng.random() < 0.5}
    if kind == "mix":
        while True:
            T, K, M = _logint(rng, 1, 16384), _logint(rng, 128, 8192), _logint(rng, 128, 8192)
            if T * K * M <= 16384 * 4096 * 8192 and T * (K + M) <= 2 ** 27:
                break
        return {"kind": kind, "T": T, "K": K, "M": M, "dt": dt, "out": rng.choice(["bf16", "f32"]),
                "bias": rng.random() < 0.5, "relu": rng.random() < 0.3}
    while True:
        N, K, P, M = _logint(rng, 1, 32), _logint(rng, 64, 2048), _logint(rng, 64, 8192), _logint(rng, 32, 1024)
        if N * P * (K + M) <= 2 ** 27 + 2 ** 25:
            break
    return {"kind": kind, "N": N, "K": K, "P": P, "M": M, "dt": dt, "out": rng.choice(["bf16", "f32"]),
            "bias": rng.random() < 0.5, "relu": rng.random() < 0.5}


# ---- inputs -----------------------------------------------------------------

def _gen(seed, tag):
    return torch.Generator(device=DEVICE).manual_seed((int(seed) * 1000003 + tag) & 0x7fffffff)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _gate(g, form, *shape):
    """Gate values of a trained layer: memories from a few steps to thousands,
    with a hard reset now and then (the start of another document)."""
    v = _randn(g, *shape).mul_(2.0).add_(3.0)
    reset = torch.rand(shape, generator=g, device=DEVICE) < 1.0 / 1024
    if form == "value":
        return torch.sigmoid(v).masked_fill_(reset, 0.0)
    return v.masked_fill_(reset, -float("inf"))


def _lengths(g, N, T):
    n = torch.randint(0, T + 1, (N,), generator=g, device=DEVICE, dtype=torch.int32)
    n[0] = T
    if N > 1:
        n[N // 2] = 0
    return n


def _seq_shape(case, C):
    return (case["N"], case["T"], C) if case["layout"] == "tokens" else (case["N"], C, case["T"])


def _halves(case, t):
    C, dim = case["C"], 2 if case["layout"] == "tokens" else 1
    return t.narrow(dim, 0, C), t.narrow(dim, C, C)


def _scan_inputs(case, seed):
    g, dt, C, N = _gen(seed, 1), _DT[case["dt"]], case["C"], case["N"]
    shape = _seq_shape(case, C)
    d = {"gate": _gate(g, case["form"], *shape).to(dt), "x": _randn(g, *shape).to(dt)}
    if case["packed"]:
        p = torch.cat([d["gate"], d["x"]], dim=2 if case["layout"] == "tokens" else 1)
        d["gate"], d["x"] = _halves(case, p)
    d["h0"] = _randn(g, N, C) if case["start"] else None
    d["lengths"] = _lengths(g, N, case["T"]) if case["ragged"] else None
    if case["kind"] == "train":
        d["dy"] = _randn(g, *shape).to(dt)
        d["dh"] = _randn(g, N, C)
    return d


def _step_inputs(case, seed):
    g, dt, C, N = _gen(seed, 2), _DT[case["dt"]], case["C"], case["N"]
    d = {"gate": _gate(g, case["form"], N, C).to(dt), "x": _randn(g, N, C).to(dt),
         "pool": _randn(g, case["S"], C),
         "slots": torch.randperm(case["S"], generator=g, device=DEVICE)[:N].to(torch.int32)}
    if N > 16:   # idle rows of the batch
        d["slots"][torch.rand(N, generator=g, device=DEVICE) < 0.05] = -1
    return d


def _codes(v):
    """Codes (as fp32 integers) and scales of the rows of v, by the definition."""
    m = v.abs().amax(dim=-1, keepdim=True)
    live = m >= _TINY
    top = torch.full_like(m, 127.0)   # a tensor: number / tensor is a reciprocal and a product, two roundings
    inv = torch.where(live, top / torch.where(live, m, torch.ones_like(m)), torch.zeros_like(m))
    return torch.round(v * inv), torch.where(live, m / 127.0, torch.zeros_like(m))


def _pitch(K):
    if own:
        from paper_1906_11367_amd import boxconv as bc
        return bc.i8_pitch(K)
    return (K + 127) // 128 * 128


def _mix_inputs(case, seed):
    g, dt, K, M = _gen(seed, 3), _DT[case["dt"]], case["K"], case["M"]
    w = _randn(g, M, K) / math.sqrt(K)
    wq, ws = _codes(w)
    d = {"wq": torch.zeros((M, _pitch(K)), dtype=torch.int8, device=DEVICE), "ws": ws.reshape(M).contiguous()}
    d["wq"][:, :K] = wq.to(torch.int8)
    if case["kind"] == "mix":
        # activations: each token at its own level, a few channels far above the
        # rest, and padding tokens of zeros
        T = case["T"]
        x = _randn(g, T, K) * torch.exp(_randn(g, T, 1)) * torch.exp(0.7 * _randn(g, 1, K))
        if T > 16:
            x[torch.rand(T, generator=g, device=DEVICE) < 0.02] = 0.0
    else:
        x = _randn(g, case["N"], K, case["P"]).mul_(torch.exp(0.5 * _randn(g, case["N"], K, 1)))
    d["x"] = x.to(dt)
    d["bias"] = _randn(g, M) if case["bias"] else None
    return d


def prepare(case, seed):
    st = {"case": dict(case)}
    kind = case["kind"]
    if kind == "step":
        st.update(_step_inputs(case, seed))
        # the pool that takes the new states (the old ones stay, so that a token
        # can be taken back); one row more than a server has, for the plain form
        st["grown"] = torch.cat([st["pool"], st["pool"][:1]])
        st["y"] = torch.empty((case["N"], case["C"]), dtype=_DT[case["dt"]], device=DEVICE)
        return st
    if kind in ("mix", "maps"):
        st.update(_mix_inputs(case, seed))
        shape = (case["T"], case["M"]) if kind == "mix" else (case["N"], case["M"], case["P"])
        st["out"] = torch.empty(shape, dtype=_DT[case["out"]], device=DEVICE)
        if own:
            from paper_1906_11367_amd import boxconv as bc
            layout = bc.BC_TOKENS if kind == "mix" else bc.BC_MAPS
            n = bc.mix_i8_workspace_bytes(case.get("N", 1), case["M"], case["K"],
                                          case["T"] if kind == "mix" else case["P"], bc.dtype_code(st["x"]), layout)
            st["wsp"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)
        return st
    st.update(_scan_inputs(case, seed))
    N, T, C, dt = case["N"], case["T"], case["C"], _DT[case["dt"]]
    shape = _seq_shape(case, C)
    st["y"] = torch.empty(shape, dtype=dt, device=DEVICE)
    st["h_last"] = torch.empty((N, C), device=DEVICE)
    if kind == "train":
        if case["packed"]:   # one buffer, as the projection's backward reads it
            st["dgate"], st["dx"] = _halves(case, torch.empty(_seq_shape(case, 2 * C), dtype=dt, device=DEVICE))
        else:
            st["dgate"], st["dx"] = (torch.empty(shape, dtype=dt, device=DEVICE) for _ in range(2))
        st["dh0"] = torch.empty((N, C), device=DEVICE) if case["start"] else None
    if own:
        from paper_1906_11367_amd import boxconv as bc
        layout = bc.BC_TOKENS if case["layout"] == "tokens" else bc.BC_MAPS
        n = max(bc.gated_scan_workspace_bytes(op, N, T, C, bc.dtype_code(st["x"]), layout)
                for op in ((0, 1) if kind == "train" else (0,)))
        st["wsp"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)
        st["states"] = bc.gated_scan_states(N, T, C, st["x"].dtype, layout, DEVICE) if kind == "train" else None
    return st


# ---- the passes -------------------------------------------------------------

def _run_own(st):
    from paper_1906_11367_amd import boxconv as bc
    case = st["case"]
    kind = case["kind"]
    if kind in ("mix", "maps"):
        return bc.pointwise_mix_i8(st["wq"], st["ws"], st["x"], st["out"],
                                   layout=bc.BC_TOKENS if kind == "mix" else bc.BC_MAPS, bias=st["bias"],
                                   relu=int(case["relu"]), ws=st["wsp"])
    form = bc.BC_GATE_LOGIT if case["form"] == "logit" else bc.BC_GATE_VALUE
    if kind == "step":
        new = st["grown"][:case["S"]]
        bc.gated_scan_step(st["gate"], st["x"], st["pool"], st["y"], slots=st["slots"], state_out=new, form=form)
        return st["y"], new
    layout = bc.BC_TOKENS if case["layout"] == "tokens" else bc.BC_MAPS
    bc.gated_scan_fwd(st["gate"], st["x"], st["y"], h0=st["h0"], h_last=st["h_last"], lengths=st["lengths"],
                      states=st["states"], form=form, layout=layout, ws=st["wsp"])
    out = {"y": st["y"], "h_last": st["h_last"]}
    if kind == "train":
        bc.gated_scan_bwd(st["gate"], st["x"], st["states"], st["dy"], st["dgate"], st["dx"], grad_h_last=st["dh"],
                          grad_h0=st["dh0"], lengths=st["lengths"], form=form, layout=layout, ws=st["wsp"])
        out.update(dgate=st["dgate"], dx=st["dx"])
        if case["start"]:
            out["dh0"] = st["dh0"]
    return out


def _coefficients(gate, x, form):
    """a and b of h_t = a_t h_{t-1} + b_t, in 32 bits."""
    gate, x = gate.float(), x.float()
    if form == "value":
        return gate, x
    e = torch.exp(-gate.abs())
    r = 1.0 / (1.0 + e)
    a, rest = torch.where(gate >= 0, r, e * r), torch.where(gate >= 0, e * r, r)
    return a, rest * x


def _prefix(a, b, dim):
    """All states of the recurrence by doubling: pairs (a, b) of ever longer runs."""
    a, b, n, s = a.clone(), b.clone(), a.shape[dim], 1
    while s < n:
        lo_a, lo_b, hi_a = a.narrow(dim, 0, n - s), b.narrow(dim, 0, n - s), a.narrow(dim, s, n - s)
        add, mul = hi_a * lo_b, hi_a * lo_a
        b.narrow(dim, s, n - s).add_(add)
        hi_a.copy_(mul)
        s *= 2
    return b


def _run_plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "mix":
        q, s = _codes(st["x"].float())
        K = case["K"]
        z = (q @ st["wq"][:, :K].float().t()) * s * st["ws"]
        if st["bias"] is not None:
            z = z + st["bias"]
        return (torch.relu(z) if case["relu"] else z).to(_DT[case["out"]])
    if kind == "maps":
        K = case["K"]
        q, s = _codes(st["x"].float().transpose(1, 2))          # [N, P, K]
        w = st["wq"][:, :K].float().t()
        z = (q.reshape(-1, K) @ w).reshape(case["N"], case["P"], case["M"]) * s * st["ws"]
        if st["bias"] is not None:
            z = z + st["bias"]
        z = torch.relu(z) if case["relu"] else z
        return z.to(_DT[case["out"]]).transpose(1, 2).contiguous()
    if kind == "step":
        a, b = _coefficients(st["gate"], st["x"], case["form"])
        slots = st["slots"].long()
        live = slots >= 0
        h = a * st["pool"][slots.clamp(min=0)] + b
        # idle rows change no state: their target is the row past the pool
        st["grown"][torch.where(live, slots, torch.full_like(slots, case["S"]))] = h
        return torch.where(live[:, None], h, torch.zeros_like(h)).to(_DT[case["dt"]]), st["grown"][:case["S"]]
    N, T, C = case["N"], case["T"], case["C"]
    tokens = case["layout"] == "tokens"
    dim = 1 if tokens else 2
    col = (lambda v: v.unsqueeze(dim))
    a, b = _coefficients(st["gate"], st["x"], case["form"])
    live = None
    if st["lengths"] is not None:
        t = torch.arange(T, device=DEVICE)
        live = t[None, :] < st["lengths"][:, None]
        live = live[:, :, None] if tokens else live[:, None, :]
        a, b = torch.where(live, a, torch.ones_like(a)), torch.where(live, b, torch.zeros_like(b))
    if st["h0"] is not None:
        b = b.clone()
        b.narrow(dim, 0, 1).add_(a.narrow(dim, 0, 1) * col(st["h0"]))
    h = _prefix(a, b, dim)
    y = h if live is None else torch.where(live, h, torch.zeros_like(h))
    dt = _DT[case["dt"]]
    out = {"y": y.to(dt), "h_last": h.select(dim, T - 1).contiguous()}
    if kind != "train":
        return out
    dy = st["dy"].float()
    if live is not None:
        dy = torch.where(live, dy, torch.zeros_like(dy))
    # r_t = a_t (dy_t + r_{t+1}), the gradient carried to the state before t
    ar, br = a.flip(dim), (a * dy).flip(dim)
    br.narrow(dim, 0, 1).add_(ar.narrow(dim, 0, 1) * col(st["dh"]))
    r = _prefix(ar, br, dim).flip(dim)
    delta = dy + torch.cat([r.narrow(dim, 1, T - 1), col(st["dh"])], dim=dim)
    first = torch.zeros((N, C), device=DEVICE) if st["h0"] is None else st["h0"]
    before = torch.cat([col(first), h.narrow(dim, 0, T - 1)], dim=dim)
    if case["form"] == "value":
        dgate, dx = delta * before, delta
    else:
        x, gate = st["x"].float(), st["gate"].float()
        e = torch.exp(-gate.abs())
        den = 1.0 + e
        rest = torch.where(gate >= 0, e / den, 1.0 / den)
        dx = delta * rest
        dgate = delta * (before - x) * (e / (den * den))
    if live is not None:
        dgate, dx = (torch.where(live, v, torch.zeros_like(v)) for v in (dgate, dx))
    out.update(dgate=dgate.to(dt), dx=dx.to(dt))
    if case["start"]:
        out["dh0"] = r.select(dim, 0).contiguous()
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the cost of a pass, and the definition in 64 bits ----------------------

def _size(dt):
    return 2 if dt == "bf16" else 4


def work(case):
    kind, e = case["kind"], _size(case["dt"])
    if kind == "step":
        n = case["N"] * case["C"]
        return {"bytes": n * (3 * e + 8) + case["N"] * 4, "flops": 8 * n}
    if kind in ("scan", "train"):
        n, rows = case["N"] * case["T"] * case["C"], case["N"] * case["C"] * 4
        b, f = 3 * n * e + rows * (2 if case["start"] else 1), 8 * n
        if kind == "train":
            b, f = b + 5 * n * e + rows * (2 if case["start"] else 1), f + 20 * n
        return {"bytes": b, "flops": f}
    rows = case["T"] if kind == "mix" else case["N"] * case["P"]
    K, M = case["K"], case["M"]
    return {"bytes": rows * (K * e + M * _size(case["out"])) + M * (K + 4) + (4 * M if case["bias"] else 0),
            "flops": 2 * rows * K * M}


def _exact_codes(v):
    """The definition's integer codes and scales, for numpy rows of 32 bits."""
    m = np.abs(v).max(axis=1, keepdims=True).astype(np.float32)
    live = m >= np.float32(_TINY)
    safe = np.where(live, m, np.float32(1))
    inv = np.where(live, np.float32(127) / safe, np.float32(0)).astype(np.float32)
    return np.rint(v * inv), np.where(live, m / np.float32(127), np.float32(0)).astype(np.float32)


def _exact_mix(case, seed):
    d = _mix_inputs(case, seed)
    K, M = case["K"], case["M"]
    x = d["x"].float()
    rows = (x if case["kind"] == "mix" else x.transpose(1, 2).reshape(-1, K)).cpu().numpy()
    q, s = _exact_codes(rows)
    q = torch.from_numpy(q).to(DEVICE, torch.float64)
    w = d["wq"][:, :K].to(torch.float64).t().contiguous()
    z = torch.mm(q, w)
    z *= torch.from_numpy(s).to(DEVICE, torch.float64)
    z *= d["ws"].to(torch.float64)
    if d["bias"] is not None:
        z += d["bias"].to(torch.float64)
    if case["relu"]:
        z = z.clamp(min=0)
    return z if case["kind"] == "mix" else z.reshape(case["N"], case["P"], M).transpose(1, 2).contiguous()


def _exact_step(case, seed):
    d = _step_inputs(case, seed)
    g, x, state = d["gate"].double(), d["x"].double(), d["pool"].double()
    a = torch.sigmoid(g) if case["form"] == "logit" else g
    b = torch.sigmoid(-g) * x if case["form"] == "logit" else x
    y = torch.zeros_like(x)
    for n, s in enumerate(d["slots"].tolist()):
        if s >= 0:
            state[s] = a[n] * state[s] + b[n]
            y[n] = state[s]
    return y, state


def _exact_scan(case, seed):
    """One step after the other, in 64 bits, time first."""
    d = _scan_inputs(case, seed)
    N, T, C = case["N"], case["T"], case["C"]
    order, back = ((1, 0, 2), (1, 0, 2)) if case["layout"] == "tokens" else ((2, 0, 1), (1, 2, 0))
    g, x = (d[k].double().permute(order).contiguous() for k in ("gate", "x"))
    live = None
    if d["lengths"] is not None:
        live = (torch.arange(T, device=DEVICE)[:, None] < d["lengths"][None, :])[:, :, None]
    logit = case["form"] == "logit"
    a, c = (torch.sigmoid(g), torch.sigmoid(-g)) if logit else (g, torch.ones_like(g))
    b = c * x
    if live is not None:   # past its end a sequence keeps its state
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    h = torch.zeros((N, C), dtype=torch.float64, device=DEVICE) if d["h0"] is None else d["h0"].double()
    hs = torch.empty((T + 1, N, C), dtype=torch.float64, device=DEVICE)
    hs[0] = h
    for t in range(T):
        torch.addcmul(b[t], a[t], hs[t], out=hs[t + 1])
    y = hs[1:] if live is None else torch.where(live, hs[1:], 0.0)
    out = {"y": y.permute(back).contiguous(), "h_last": hs[T].clone()}
    if case["kind"] != "train":
        return out
    dy = d["dy"].double().permute(order).contiguous()
    if live is not None:
        dy = torch.where(live, dy, 0.0)
    delta = torch.empty_like(dy)
    r = d["dh"].double()
    for t in range(T - 1, -1, -1):
        torch.add(dy[t], r, out=delta[t])
        r = a[t] * delta[t]
    da = delta * hs[:-1]
    if logit:
        da = (da - delta * x) * a * c
    dx = delta * c
    if live is not None:
        da, dx = torch.where(live, da, 0.0), torch.where(live, dx, 0.0)
    out.update(dgate=da.permute(back).contiguous(), dx=dx.permute(back).contiguous())
    if case["start"]:
        out["dh0"] = r
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind in ("mix", "maps"):
        return _exact_mix(case, seed)
    return _exact_step(case, seed) if kind == "step" else _exact_scan(case, seed)
