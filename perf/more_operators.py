"""The operators of a linear-attention block as its users call them, as measurable cases.

The block's middle is linear attention whose state forgets: every head keeps a
matrix of Dk x Dv that a token first scales by its decay and then adds its key
and value to, and that its query reads.  Around it stand norms: one before the
block, one over each head's outputs with a gate, one after the block with the
residual sum and the next block's norm behind it.  Both operators are used in
training (forward and backward) and in serving (prompts, then single tokens).

Linear attention, for every sequence n and head h, from S_{-1} = s0 (zero):
  S_t = a_t S_{t-1} + k_t v_t^T,   y_t = scale * S_t^T q_t
  kind    "seq"   the forward over whole sequences: outputs and last states
          "train" the forward and the backward: every gradient as well
          "token" one token for N sequences whose states live in a pool
  form    "logit": a = sigmoid(gate); "log": a = exp(gate); "fixed": a = exp of
          one number for each head, not learned
  Hq, Hk, Hv   heads of q, k and v, divisors of the H heads of decays, states and
          outputs: head h reads head h // (H // Hq) of q, and so on
  layout  "tokens" [N, T, H, D] or "heads" [N, H, T, D]
  packed  q, k, v and the gate are slices of one projection's rows
  ragged  every sequence has its own length (one of them zero, one full);
          outputs and gradients past it are zero, the last state is that at it
  start   an initial state is given (zero otherwise), and its gradient asked for

Block norm, for every row (token) of C channels:
  p = norm(z) * w_post within each of `groups` runs of channels (p = z for 0 groups)
  u = p * act(gate),   r = x + res_scale * u,   y = norm(r) * w_pre
  kind    "norm" the forward, "normgrad" the backward too
  norm    "rms": v / sqrt(mean(v^2) + eps); "layer": the mean is taken off first
  act     "silu", "sigmoid" or "" (no gate)
  res, rs, pre   whether there is an x, a res_scale, and a y
"""
import math

import torch

own = False
DEVICE = "cuda:0"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6
_CHUNK = 64


def _attn(name, kind, N, T, H, Dk, Dv, dt, form="logit", heads=None, layout="tokens", packed=True, ragged=False,
          start=False):
    Hq, Hk, Hv = heads or (H, H, H)
    return {"name": name, "kind": kind, "N": N, "T": T, "H": H, "Hq": Hq, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv,
            "dt": dt, "form": form, "layout": layout, "packed": packed, "ragged": ragged, "start": start}


def _token(name, N, H, Dk, Dv, S, dt, form="logit", heads=None):
    Hq, Hk, Hv = heads or (H, H, H)
    return {"name": name, "kind": "token", "N": N, "H": H, "Hq": Hq, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "S": S,
            "dt": dt, "form": form}


def _norm(name, kind, R, groups, size, dt, norm="rms", act="", res=False, rs=False, pre=False):
    """groups runs of `size` channels under the first norm; groups = 0: none, `size` channels."""
    return {"name": name, "kind": kind, "R": R, "C": max(groups, 1) * size, "groups": groups, "dt": dt, "norm": norm,
            "act": act, "res": res, "rs": rs, "pre": pre}


def listed():
    return [
        # one new token for a handful of sequences: latency only
        _token("token_4", 4, 8, 64, 64, 8, "bf16"),
        # a full serving batch, its states scattered in a pool, a few rows idle
        _token("token_128", 128, 16, 128, 128, 192, "bf16"),
        # a batch of short prompts, padded, keys and values shared by four heads
        _attn("prompts", "seq", 16, 200, 16, 64, 64, "bf16", heads=(16, 4, 4), ragged=True),
        # one long document: few heads, all the work along the time axis
        _attn("document", "seq", 1, 65536, 8, 128, 128, "bf16", start=True),
        # the operator in training on token sequences
        _attn("train_tokens", "train", 4, 4096, 16, 128, 128, "bf16"),
        # the same on few long sequences with decays that are not learned, in fp32, heads outermost
        _attn("train_fixed", "train", 1, 8192, 8, 64, 128, "f32", form="fixed", layout="heads", packed=False),
        # odd sizes, padded sequences, shared queries and keys, coefficients given as logarithms
        _attn("train_ragged", "train", 3, 1531, 6, 40, 72, "f32", form="log", heads=(2, 2, 6), packed=False, ragged=True,
              start=True),
        # the norm before a block for a handful of tokens: latency only
        _norm("norm_8", "norm", 8, 0, 1024, "bf16", pre=True),
        # each head's outputs normed and gated, a prefill batch
        _norm("norm_heads", "norm", 16384, 16, 128, "bf16", act="silu"),
        # the same in training
        _norm("norm_heads_train", "normgrad", 16384, 16, 128, "bf16", act="silu"),
        # after a wide block in training: norm, residual with its scale, the next block's norm
        _norm("norm_block_train", "normgrad", 8192, 1, 4096, "bf16", res=True, rs=True, pre=True),
        # odd sizes everywhere, everything at once, fp32
        _norm("norm_odd_train", "normgrad", 777, 3, 279, "f32", norm="layer", act="sigmoid", res=True, rs=True, pre=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng):
    H = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    share = [d for d in (1, 2, 3, 4, 6, 8, 12, 16) if H % d == 0]
    return H, [H if rng.random() < 0.6 else rng.choice(share) for _ in range(3)]


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    kind = rng.choice(["seq", "train", "train", "token", "norm", "normgrad"])
    dt = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "normgrad"):
        while True:
            R, groups, size = _logint(rng, 1, 32768), rng.choice([0, 0, 1, 1, 3, 8, 16, 20]), _logint(rng, 24, 8192)
            C = max(groups, 1) * size
            if 64 <= C <= 8192 and R * C <= 2 ** 25:
                break
        if rng.random() < 0.6:   # whole vectors
            size = (size + 7) // 8 * 8
            while max(groups, 1) * size > 8192:
                size -= 8
        res = rng.random() < 0.6
        return _norm("", kind, R, groups, size, dt, rng.choice(["rms", "rms", "layer"]),
                     rng.choice(["", "silu", "sigmoid"]), res, rng.random() < 0.5,
                     rng.random() < 0.6 or not (groups or res))
    form = rng.choice(["logit", "logit", "log", "fixed"])
    H, heads = _draw_heads(rng)
    Dk, Dv = (rng.choice([64, 128]) if rng.random() < 0.6 else rng.randint(8, 128) for _ in range(2))
    if kind == "token":
        N = _logint(rng, 1, max(1, 128 * 16 // H))
        return _token("", N, H, Dk, Dv, N + _logint(rng, 1, 64), dt, form, heads)
    while True:
        N, T = _logint(rng, 1, 64), _logint(rng, 1, 65536 if kind == "seq" else 16384)
        if N * T * H * (Dk + Dv) <= 2 ** (26 if dt == "bf16" else 25) and N * T * H >= 64:
            break
    layout = rng.choice(["tokens", "tokens", "heads"])
    packed = layout == "tokens" and rng.random() < 0.5
    if packed:   # slices of one projection: whole vectors of 16 bytes
        Dk, Dv = (max(8, D // 8 * 8) for D in (Dk, Dv))
    return _attn("", kind, N, T, H, Dk, Dv, dt, form, heads, layout, packed, rng.random() < 0.4,
                 rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------

def _gen(seed, tag):
    return torch.Generator(device=DEVICE).manual_seed((int(seed) * 1000003 + tag) & 0x7fffffff)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _gate(g, case, *shape):
    """Gates of a trained layer: memories from a few steps to thousands, with a
    hard reset now and then (the start of another document); or one logarithm
    for each head, memories of 32 steps and more."""
    if case["form"] == "fixed":
        H = case["H"]
        return torch.log1p(-torch.exp2(-5.0 - 7.0 * torch.arange(H, device=DEVICE) / H))
    v = _randn(g, *shape).mul_(2.0).add_(3.0)
    if case["form"] == "log":
        v = torch.minimum(v, torch.zeros_like(v)) - torch.log1p(torch.exp(-v.abs()))
    return v.masked_fill_(torch.rand(shape, generator=g, device=DEVICE) < 1.0 / 1024, -float("inf")).to(_DT[case["dt"]])


def _lengths(g, N, T):
    n = torch.randint(0, T + 1, (N,), generator=g, device=DEVICE, dtype=torch.int32)
    n[0] = T
    if N > 1:
        n[N // 2] = 0
    return n


def _shaped(case, H, D, make):
    """A tensor [N, T, H, D] of the case's layout; make(*shape) gives it dense."""
    N, T = case["N"], case["T"]
    return make(N, T, H, D) if case["layout"] == "tokens" else make(N, H, T, D).transpose(1, 2)


def _empty(dt):
    return lambda *shape: torch.empty(shape, dtype=dt, device=DEVICE)


def _packed_split(case, rows):
    """q, k, v and the gate (none where it is fixed) out of rows [N, T, ...]."""
    at, out = 0, []
    for H, D in ((case["Hq"], case["Dk"]), (case["Hk"], case["Dk"]), (case["Hv"], case["Dv"])):
        out.append(rows[:, :, at:at + H * D].unflatten(2, (H, D)))
        at += H * D
    return out, (rows[:, :, at:at + case["H"]] if case["form"] != "fixed" else None)


def _packed_width(case):
    n = (case["Hq"] + case["Hk"]) * case["Dk"] + case["Hv"] * case["Dv"]
    return n + ((case["H"] + 7) // 8 * 8 if case["form"] != "fixed" else 0)


def _attn_inputs(case, seed):
    g, dt = _gen(seed, 1), _DT[case["dt"]]
    N, T, H, Dk, Dv = (case[k] for k in ("N", "T", "H", "Dk", "Dv"))
    make = lambda *shape: _randn(g, *shape).to(dt)
    gate = _gate(g, case, N, T, H)
    if case["packed"]:
        rows = make(N, T, _packed_width(case))
        (q, k, v), at = _packed_split(case, rows)
        if at is not None:
            at.copy_(gate)
            gate = at
    else:
        q, k, v = (_shaped(case, h, d, make) for h, d in ((case["Hq"], Dk), (case["Hk"], Dk), (case["Hv"], Dv)))
    d = {"q": q, "k": k, "v": v, "gate": gate,
         "s0": _randn(g, N, H, Dk, Dv) if case["start"] else None,
         "lengths": _lengths(g, N, T) if case["ragged"] else None}
    if case["kind"] == "train":
        d["dy"] = _shaped(case, H, Dv, make)
        d["ds"] = _randn(g, N, H, Dk, Dv)
    return d


def _token_inputs(case, seed):
    g, dt = _gen(seed, 2), _DT[case["dt"]]
    N, H, Dk, Dv, S = (case[k] for k in ("N", "H", "Dk", "Dv", "S"))
    d = {"q": _randn(g, N, case["Hq"], Dk).to(dt), "k": _randn(g, N, case["Hk"], Dk).to(dt),
         "v": _randn(g, N, case["Hv"], Dv).to(dt), "gate": _gate(g, case, N, H), "pool": _randn(g, S, H, Dk, Dv),
         "slots": torch.randperm(S, generator=g, device=DEVICE)[:N].to(torch.int32)}
    if N > 16:   # idle rows of the batch
        d["slots"][torch.rand(N, generator=g, device=DEVICE) < 0.05] = -1
    return d


def _norm_inputs(case, seed):
    """Rows at their own levels with a few channels far above the rest, and rows
    of zeros (padding)."""
    g, dt, R, C = _gen(seed, 3), _DT[case["dt"]], case["R"], case["C"]
    level = torch.exp(0.7 * _randn(g, R, 1)) * torch.exp(0.7 * _randn(g, 1, C))
    z = _randn(g, R, C) * level
    if R > 16:
        z[torch.rand(R, generator=g, device=DEVICE) < 0.02] = 0.0
    d = {"z": z.to(dt), "gate": _randn(g, R, C).mul_(1.5).to(dt) if case["act"] else None,
         "x": _randn(g, R, C).mul_(2.0).to(dt) if case["res"] else None,
         "w_post": 1.0 + 0.2 * _randn(g, C) if case["groups"] else None,
         "res_scale": 0.5 + 0.2 * _randn(g, C) if case["rs"] else None,
         "w_pre": 1.0 + 0.2 * _randn(g, C) if case["pre"] else None}
    if case["kind"] == "normgrad":
        d["dr"] = _randn(g, R, C).to(dt)
        d["dy"] = _randn(g, R, C).to(dt) if case["pre"] else None
    return d


def prepare(case, seed):
    st = {"case": dict(case)}
    kind, dt = case["kind"], _DT[case["dt"]]
    if kind == "token":
        st.update(_token_inputs(case, seed))
        # the pool that takes the new states (the old ones stay, so that a token
        # can be taken back); one row more than a server has, for the plain form
        st["grown"] = torch.cat([st["pool"], st["pool"][:1]])
        st["y"] = _empty(dt)(case["N"], case["H"], case["Dv"])
        return st
    if kind in ("norm", "normgrad"):
        st.update(_norm_inputs(case, seed))
        R, C = case["R"], case["C"]
        new = _empty(dt)
        st["r"], st["y"] = new(R, C), new(R, C) if case["pre"] else None
        if kind == "normgrad":
            for name in ("z", "gate", "x"):
                st["d" + name] = new(R, C) if st[name] is not None else None
            for name in ("w_post", "res_scale", "w_pre"):
                st["d" + name] = _empty(torch.float32)(C) if st[name] is not None else None
            if own:
                from paper_1906_11367_amd import boxconv as bc
                st["ws"] = _empty(torch.uint8)(max(bc.block_norm_workspace_bytes(R, C), 16))
        return st
    st.update(_attn_inputs(case, seed))
    N, T, H, Dk, Dv = (case[k] for k in ("N", "T", "H", "Dk", "Dv"))
    st["y"], st["s_last"] = _shaped(case, H, Dv, _empty(dt)), _empty(torch.float32)(N, H, Dk, Dv)
    if kind == "train":
        if case["packed"]:   # one buffer, as the projection's backward reads it
            rows = torch.zeros((N, T, _packed_width(case)), dtype=dt, device=DEVICE)
            (st["dq"], st["dk"], st["dv"]), st["dgate"] = _packed_split(case, rows)
        else:
            st["dq"], st["dk"], st["dv"] = (_shaped(case, h, d, _empty(dt)) for h, d in
                                            ((case["Hq"], Dk), (case["Hk"], Dk), (case["Hv"], Dv)))
            st["dgate"] = _empty(dt)(N, T, H) if case["form"] != "fixed" else None
        st["ds0"] = _empty(torch.float32)(N, H, Dk, Dv) if case["start"] else None
    if own:
        from paper_1906_11367_amd import boxconv as bc
        sizes = (N, T, H, case["Hq"], case["Hk"], case["Hv"], Dk, Dv, bc.dtype_code(st["q"]))
        n = max(bc.linear_attention_workspace_bytes(op, *sizes) for op in ((0, 1) if kind == "train" else (0,)))
        st["ws"] = _empty(torch.uint8)(max(n, 16))
        st["states"] = bc.linear_attention_states(N, T, H, Dk, Dv, DEVICE) if kind == "train" else None
    return st


# ---- the passes -------------------------------------------------------------

def _scale(case):
    return case["Dk"] ** -0.5


def _run_own(st):
    from paper_1906_11367_amd import boxconv as bc
    case = st["case"]
    kind = case["kind"]
    if kind in ("norm", "normgrad"):
        how = dict(groups=case["groups"], kind=bc.BC_NORM_RMS if case["norm"] == "rms" else bc.BC_NORM_LAYER,
                   act=bc.BC_ACT_SIGMOID if case["act"] == "sigmoid" else bc.BC_ACT_SILU, eps=_EPS)
        params = dict(gate=st["gate"], x=st["x"], w_post=st["w_post"], res_scale=st["res_scale"], w_pre=st["w_pre"])
        bc.block_norm_fwd(st["z"], r=st["r"], y=st["y"], **params, **how)
        out = {"r": st["r"]}
        if case["pre"]:
            out["y"] = st["y"]
        if kind == "normgrad":
            names = ("z", "gate", "x", "w_post", "res_scale", "w_pre")
            grads = {"grad_" + n: st["d" + n] for n in names}
            bc.block_norm_bwd(st["z"], grad_r=st["dr"], grad_y=st["dy"], ws=st["ws"], **params, **grads, **how)
            out.update({"d" + n: st["d" + n] for n in names if st["d" + n] is not None})
        return out
    form = bc.BC_GATE_LOGIT if case["form"] == "logit" else bc.BC_GATE_LOG
    if kind == "token":
        new = st["grown"][:case["S"]]
        bc.linear_attention_step(st["q"], st["k"], st["v"], st["gate"], st["pool"], st["y"], slots=st["slots"],
                                 state_out=new, form=form, scale=_scale(case))
        return st["y"], new
    how = dict(lengths=st["lengths"], form=form, scale=_scale(case), ws=st["ws"])
    bc.linear_attention_fwd(st["q"], st["k"], st["v"], st["gate"], st["y"], s0=st["s0"], s_last=st["s_last"],
                            states=st["states"], **how)
    out = {"y": st["y"], "s_last": st["s_last"]}
    if kind == "train":
        bc.linear_attention_bwd(st["q"], st["k"], st["v"], st["gate"], st["states"], st["dy"], st["dq"], st["dk"],
                                st["dv"], st["dgate"], grad_s_last=st["ds"], grad_s0=st["ds0"], **how)
        out.update({n: st[n] for n in ("dq", "dk", "dv", "dgate", "ds0") if st[n] is not None})
    return out


def _log_decay(gate, form):
    """The logarithms of the decays, in 64 bits (their sums over a chunk lose
    digits in 32); what is left of a state after e^-10000 is nothing."""
    g = gate.double()
    if form == "logit":
        g = torch.minimum(g, torch.zeros_like(g)) - torch.log1p(torch.exp(-g.abs()))
    return g.clamp(min=-1e4)


def _plain_token(st):
    case = st["case"]
    H = case["H"]
    q, k, v = (st[n].float().repeat_interleave(H // st[n].shape[1], dim=1) for n in ("q", "k", "v"))
    a = torch.exp(_log_decay(st["gate"], case["form"])).float()
    slots = st["slots"].long()
    live = slots >= 0
    s = a[..., None, None] * st["pool"][slots.clamp(min=0)] + k[..., :, None] * v[..., None, :]
    # idle rows change no state: their target is the row past the pool
    st["grown"][torch.where(live, slots, torch.full_like(slots, case["S"]))] = s
    y = (q[..., :, None] * s).sum(dim=-2) * _scale(case)
    return torch.where(live[:, None, None], y, torch.zeros_like(y)).to(_DT[case["dt"]]), st["grown"][:case["S"]]


def _plain_attention(st):
    """In chunks of 64 tokens: with L the running sum of the logarithms within a
    chunk, token j reaches token i of its chunk by exp(L_i - L_j), the chunk's
    end by exp(L_end - L_j), and the state before the chunk reaches i by exp(L_i)."""
    case = st["case"]
    N, T, H, Dk, Dv, dt = *(case[k] for k in ("N", "T", "H", "Dk", "Dv")), _DT[case["dt"]]
    nch = (T + _CHUNK - 1) // _CHUNK
    live = None
    if st["lengths"] is not None:
        live = torch.arange(T, device=DEVICE)[None, :] < st["lengths"][:, None]

    def chunks(t):   # [N, T, heads, D] -> [N * H, nch, 64, D] in 32 bits, zero past the end
        t = t.float()
        if live is not None:
            t = torch.where(live[:, :, None, None], t, torch.zeros_like(t))
        t = t.repeat_interleave(H // t.shape[2], dim=2)
        t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, nch * _CHUNK - T))
        return t.permute(0, 2, 1, 3).reshape(N * H, nch, _CHUNK, -1).contiguous()

    def tokens(t, heads):   # the way back, the heads that share summed
        t = t.reshape(N, H, nch * _CHUNK, -1)[:, :, :T].permute(0, 2, 1, 3)
        if heads != H:
            t = t.unflatten(2, (heads, H // heads)).sum(dim=3)
        return t.to(dt).contiguous()

    log = _log_decay(st["gate"], case["form"]).expand(N, T, H)
    if live is not None:
        log = torch.where(live[:, :, None], log, torch.zeros_like(log))
    log = torch.nn.functional.pad(log, (0, 0, 0, nch * _CHUNK - T))
    L = log.permute(0, 2, 1).reshape(N * H, nch, _CHUNK).cumsum(dim=2)
    end = L[:, :, -1:]
    here, rest, whole = (torch.exp(v).float()[..., None] for v in (L, end - L, end))
    before = torch.ones((_CHUNK, _CHUNK), dtype=torch.bool, device=DEVICE).tril()
    reach = torch.exp((L[..., :, None] - L[..., None, :]).masked_fill(~before, -float("inf"))).float()

    scale = _scale(case)
    q, k, v = chunks(st["q"]) * scale, chunks(st["k"]), chunks(st["v"])
    add = (k * rest).transpose(2, 3) @ v
    S = torch.empty((nch + 1, N * H, Dk, Dv), device=DEVICE)
    S[0] = 0.0 if st["s0"] is None else st["s0"].reshape(N * H, Dk, Dv)
    for c in range(nch):
        torch.addcmul(add[:, c], whole[:, c], S[c], out=S[c + 1])
    first = S[:nch].transpose(0, 1)
    P = (q @ k.transpose(2, 3)) * reach
    out = {"y": tokens(P @ v + (q * here) @ first, H), "s_last": S[nch].reshape(N, H, Dk, Dv).clone()}
    if case["kind"] != "train":
        return out

    dy = chunks(st["dy"])
    add = (q * here).transpose(2, 3) @ dy
    dS = torch.empty((nch + 1, N * H, Dk, Dv), device=DEVICE)   # dS[c + 1]: at the end of chunk c
    dS[nch] = st["ds"].reshape(N * H, Dk, Dv)
    for c in range(nch - 1, -1, -1):
        torch.addcmul(add[:, c], whole[:, c], dS[c + 1], out=dS[c])
    last = dS[1:].transpose(0, 1)
    dP = (dy @ v.transpose(2, 3)) * reach
    dq = dP @ k + here * (dy @ first.transpose(2, 3))
    dk = dP.transpose(2, 3) @ q + rest * (v @ last.transpose(2, 3))
    dv = P.transpose(2, 3) @ dy + rest * (k @ last)
    out.update(dq=tokens(dq * scale, case["Hq"]), dk=tokens(dk, case["Hk"]), dv=tokens(dv, case["Hv"]))
    if case["form"] != "fixed":
        # what crosses the border before token t: this chunk's queries from t on
        # less its keys from t on, and all that crosses the chunk's end
        cross = ((q * dq).sum(dim=3) - (k * dk).sum(dim=3)).double()
        cross = cross.flip(2).cumsum(dim=2).flip(2)
        cross = cross + (S[1:] * dS[1:]).sum(dim=(2, 3)).transpose(0, 1)[..., None].double()
        cross = cross.reshape(N, H, nch * _CHUNK)[:, :, :T].permute(0, 2, 1).float()
        g = st["gate"].float()
        if case["form"] == "logit":
            e = torch.exp(-g.abs())
            cross = cross * torch.where(g >= 0, e, torch.ones_like(e)) / (1.0 + e)
        dead = g == -float("inf")
        if live is not None:
            dead = dead | ~live[:, :, None]
        out["dgate"] = cross.masked_fill(dead, 0.0).to(dt)
    if case["start"]:
        out["ds0"] = dS[0].reshape(N, H, Dk, Dv).clone()
    return out


def _stats(v, norm, groups):
    """v normed within groups [R, groups, size], and 1 / its deviation."""
    v = v.unflatten(1, (groups, -1))
    if norm == "layer":
        v = v - v.mean(dim=2, keepdim=True)
    rho = 1.0 / torch.sqrt((v * v).mean(dim=2, keepdim=True) + _EPS)
    return v * rho, rho


def _norm_grad(n, rho, dn, norm):
    """The gradient through n = norm(v), given that to n."""
    dn = dn.unflatten(1, n.shape[1:])
    g = dn - n * (n * dn).mean(dim=2, keepdim=True)
    if norm == "layer":
        g = g - dn.mean(dim=2, keepdim=True)
    return (g * rho).flatten(1)


def _plain_norm(st):
    case = st["case"]
    norm, groups, dt = case["norm"], case["groups"], _DT[case["dt"]]
    p = st["z"].float()
    if groups:
        n1, rho1 = _stats(p, norm, groups)
        p = n1.flatten(1) * st["w_post"]
    u = p
    if case["act"]:
        g = st["gate"].float()
        sig = 1.0 / (1.0 + torch.exp(-g))
        phi = g * sig if case["act"] == "silu" else sig
        u = p * phi
    r = u if st["res_scale"] is None else u * st["res_scale"]
    if case["res"]:
        r = st["x"].float() + r
    out = {"r": r.to(dt)}
    if case["pre"]:
        n2, rho2 = _stats(r, norm, 1)
        out["y"] = (n2.flatten(1) * st["w_pre"]).to(dt)
    if case["kind"] == "norm":
        return out
    dr = st["dr"].float()
    if case["pre"]:
        dy = st["dy"].float()
        out["dw_pre"] = (dy * n2.flatten(1)).sum(dim=0)
        dr = dr + _norm_grad(n2, rho2, dy * st["w_pre"], norm)
    if case["res"]:
        out["dx"] = dr.to(dt)
    du = dr
    if st["res_scale"] is not None:
        out["dres_scale"] = (dr * u).sum(dim=0)
        du = dr * st["res_scale"]
    dp = du
    if case["act"]:
        slope = sig * (1.0 + g * (1.0 - sig)) if case["act"] == "silu" else sig * (1.0 - sig)
        out["dgate"] = (du * p * slope).to(dt)
        dp = du * phi
    if groups:
        out["dw_post"] = (dp * n1.flatten(1)).sum(dim=0)
        dp = _norm_grad(n1, rho1, dp * st["w_post"], norm)
    out["dz"] = dp.to(dt)
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "token":
        return _plain_token(state)
    return _plain_norm(state) if kind in ("norm", "normgrad") else _plain_attention(state)


# ---- the cost of a pass, and the definition in 64 bits ----------------------

def work(case):
    kind, e = case["kind"], 2 if case["dt"] == "bf16" else 4
    if kind in ("norm", "normgrad"):
        n, C = case["R"] * case["C"], case["C"]
        ins = 1 + bool(case["act"]) + case["res"]
        params = (case["groups"] > 0) + case["rs"] + case["pre"]
        b, f = n * e * (ins + 1 + case["pre"]) + params * 4 * C, n * 12
        if kind == "normgrad":
            b, f = b + n * e * (2 * ins + 1 + case["pre"]) + 2 * params * 4 * C, f + n * 30
        return {"bytes": b, "flops": f}
    N, H, Dk, Dv = (case[k] for k in ("N", "H", "Dk", "Dv"))
    qkv, y, cell = (case["Hq"] + case["Hk"]) * Dk + case["Hv"] * Dv, H * Dv, Dk * Dv
    gate = 0 if case["form"] == "fixed" else H
    if kind == "token":
        return {"bytes": N * ((qkv + gate + y) * e + H * cell * 8 + 4), "flops": N * H * cell * 5}
    rows = N * case["T"]
    read = rows / 2 if case["ragged"] else rows       # past an end nothing need be read
    state = N * H * cell * 4 * (2 if case["start"] else 1)
    b, f = read * (qkv + gate) * e + rows * y * e + state, read * H * cell * 4
    if kind == "train":
        b += read * (qkv + gate + y) * e + rows * (qkv + gate) * e + state
        f += read * H * cell * 10
    return {"bytes": int(b), "flops": int(f)}


def _exact_decay(gate, form):
    return torch.sigmoid(gate.double()) if form == "logit" else torch.exp(gate.double())


def _exact_token(case, seed):
    d = _token_inputs(case, seed)
    H, state = case["H"], d["pool"].double()
    a = _exact_decay(d["gate"], case["form"]).expand(case["N"], H)
    y = torch.zeros((case["N"], H, case["Dv"]), dtype=torch.float64, device=DEVICE)
    of = lambda t, n: t[n].double()[torch.arange(H, device=DEVICE) // (H // t.shape[1])]
    for n, s in enumerate(d["slots"].tolist()):
        if s >= 0:
            state[s] = a[n, :, None, None] * state[s] + of(d["k"], n)[:, :, None] * of(d["v"], n)[:, None, :]
            y[n] = (of(d["q"], n)[:, :, None] * state[s]).sum(dim=1) * _scale(case)
    return y, state


def _exact_attention(case, seed):
    """One token after the other, in 64 bits, time first."""
    if case["kind"] == "train" and case["T"] > 20000:
        return None
    d = _attn_inputs(case, seed)
    N, T, H, Dk, Dv = (case[k] for k in ("N", "T", "H", "Dk", "Dv"))
    train, c = case["kind"] == "train", _scale(case)
    of = lambda t: t.double().transpose(0, 1)[:, :, torch.arange(H, device=DEVICE) // (H // t.shape[2])].contiguous()
    q, k, v = of(d["q"]), of(d["k"]), of(d["v"])
    a = _exact_decay(d["gate"], case["form"]).expand(N, T, H).transpose(0, 1).contiguous()
    dy = of(d["dy"]) if train else None
    live = None
    if d["lengths"] is not None:   # past its end a sequence keeps its state
        live = (torch.arange(T, device=DEVICE)[:, None] < d["lengths"][None, :])[:, :, None]
        a = torch.where(live, a, 1.0)
        q, k, v = (torch.where(live[..., None], t, 0.0) for t in (q, k, v))
        dy = torch.where(live[..., None], dy, 0.0) if train else None

    def grow(S, t):
        return torch.addcmul(k[t][..., :, None] * v[t][..., None, :], a[t][..., None, None], S)

    s0 = torch.zeros((N, H, Dk, Dv), dtype=torch.float64, device=DEVICE) if d["s0"] is None else d["s0"].double()
    S, y, kept = s0, torch.empty((T, N, H, Dv), dtype=torch.float64, device=DEVICE), []
    for t in range(T):
        if train and t % 64 == 0:
            kept.append(S)
        S = grow(S, t)
        y[t] = torch.matmul(q[t][..., None, :], S)[..., 0, :]
    out = {"y": y.mul_(c).transpose(0, 1), "s_last": S}
    if not train:
        return out
    dq, dk, dv, da = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(a)
    dS = d["ds"].double()
    for b in range(len(kept) - 1, -1, -1):
        run = [kept[b]]
        for t in range(64 * b, min(T, 64 * b + 64)):
            run.append(grow(run[-1], t))
        for t in range(min(T, 64 * b + 64) - 1, 64 * b - 1, -1):
            now, prior = run[t - 64 * b + 1], run[t - 64 * b]
            dS = torch.addcmul(dS, q[t][..., :, None], c * dy[t][..., None, :])
            dq[t] = c * torch.matmul(now, dy[t][..., None])[..., 0]
            dk[t] = torch.matmul(dS, v[t][..., None])[..., 0]
            dv[t] = torch.matmul(k[t][..., None, :], dS)[..., 0, :]
            da[t] = (prior * dS).sum(dim=(2, 3))
            dS = a[t][..., None, None] * dS

    def tokens(t, heads):
        t = t if live is None else torch.where(live[..., None], t, 0.0)
        return t.transpose(0, 1).unflatten(2, (heads, H // heads)).sum(dim=3)

    out.update(dq=tokens(dq, case["Hq"]), dk=tokens(dk, case["Hk"]), dv=tokens(dv, case["Hv"]))
    if case["form"] != "fixed":
        dg = da * a * (torch.sigmoid(-d["gate"].double()).transpose(0, 1) if case["form"] == "logit" else 1.0)
        out["dgate"] = (dg if live is None else torch.where(live, dg, 0.0)).transpose(0, 1)
    if case["start"]:
        out["ds0"] = dS
    return out


def _exact_norm(case, seed):
    """The definition in 64 bits, its gradients by automatic differentiation."""
    d = _norm_inputs(case, seed)
    names = [n for n in ("z", "gate", "x", "w_post", "res_scale", "w_pre") if d[n] is not None]
    leaf = {n: d[n].double().requires_grad_() for n in names}

    def norm(v):
        if case["norm"] == "layer":
            v = v - v.mean(-1, keepdim=True)
        return v * (v.square().mean(-1, keepdim=True) + _EPS).rsqrt()

    u = leaf["z"]
    if case["groups"]:
        u = norm(u.reshape(case["R"], case["groups"], -1)).reshape(u.shape) * leaf["w_post"]
    if case["act"]:
        u = u * torch.sigmoid(leaf["gate"]) * (leaf["gate"] if case["act"] == "silu" else 1.0)
    r = u * leaf["res_scale"] if case["rs"] else u
    r = r + leaf["x"] if case["res"] else r * 1.0
    out = {"r": r}
    if case["pre"]:
        out["y"] = norm(r) * leaf["w_pre"]
    if case["kind"] == "normgrad":
        loss = (r * d["dr"].double()).sum()
        if case["pre"]:
            loss = loss + (out["y"] * d["dy"].double()).sum()
        grads = torch.autograd.grad(loss, [leaf[n] for n in names])
        out.update({"d" + n: g for n, g in zip(names, grads)})
    return {n: t.detach() for n, t in out.items()}


def exact(case, seed):
    kind = case["kind"]
    if kind == "token":
        return _exact_token(case, seed)
    return _exact_norm(case, seed) if kind in ("norm", "normgrad") else _exact_attention(case, seed)
