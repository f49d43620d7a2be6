"""Linear attention with a decay for each head and the norms around its block, in
64 bits (NumPy), token by token and row by row.

Shares no code with the library.  Beside every value stands its magnitude: the
same formula with every term's absolute value.  Evaluated in 32 bits, a sum of m
terms, each the product of a few rounded factors, is off by at most about
(m + a few) * 2^-24 of its magnitude; attention_units and NORM_UNITS count them.
"""
import numpy as np

EPS = 2.0 ** -24                         # unit roundoff of fp32
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # of a value rounded to its type


def log_decay(gate, form):
    with np.errstate(over="ignore"):
        return -np.logaddexp(0.0, -gate) if form == "logit" else gate


def spread(v, H):
    """[N, T, Hx, D] -> [N, T, H, D]: head h is head h // (H // Hx)."""
    return np.repeat(v, H // v.shape[2], axis=2)


def gather(v, Hx):
    """[N, T, H, D] -> [N, T, Hx, D], the heads that share summed."""
    N, T, H, D = v.shape
    return v.reshape(N, T, Hx, H // Hx, D).sum(axis=3)


SPAN = 2048   # tokens to the border at which a sum for the gates' gradients ends, at most


def attention_units(T, Dk, Dv, dt):
    """Units of 2^-24 of the magnitudes.  Products over Dk or Dv channels, over a
    chunk's tokens (64 allowed for) and, in the state, a multiplication and an addition a chunk;
    heads that share (at most 16) and the gates' sums (q dq less k dk: twice) come on
    top; the decays' logarithms are right to a few
    units of themselves, and x e^-x < 1/2, or e^-x is small enough to lie below the
    rest.  bf16: each score, and each state that a query reads, is a sum of two bf16
    parts, off by 2^-16 or 256 units of itself.  (States themselves take in sums of three,
    2^-24: "f32" counts theirs.)"""
    c = Dk + Dv + 64 + 2 * (T // 32 + 1) + 64
    return c + (512 if dt == "bf16" else 0)


def attention(q, k, v, gate, form, scale, s0=None, lengths=None, dy=None, ds=None):
    """q [N, T, Hq, Dk], ..., gate [N, T, H] -> dict of (value, magnitude)."""
    N, T, H = gate.shape
    Hq, Hk, Hv, Dk, Dv = q.shape[2], k.shape[2], v.shape[2], q.shape[3], v.shape[3]
    n = np.full(N, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    live = np.arange(T)[None, :] < n[:, None]
    clean = lambda t: np.where(live[:, :, None, None], t, 0.0)
    q, k, v = (spread(clean(t), H) for t in (q, k, v))
    dy = None if dy is None else clean(dy)
    gate = np.where(live[:, :, None], gate, 0.0)
    a = np.where(live[:, :, None], np.exp(log_decay(gate, form)), 1.0)
    zero = np.zeros((N, H, Dk, Dv))
    S, M = (zero, zero) if s0 is None else (s0, np.abs(s0))
    y, ym = np.zeros((2, N, T, H, Dv))
    Ss, Ms = [S], [M]
    for t in range(T):
        kv = k[:, t, :, :, None] * v[:, t, :, None, :]
        S = a[:, t, :, None, None] * S + kv
        M = a[:, t, :, None, None] * M + np.abs(kv)
        y[:, t] = scale * np.einsum("nhk,nhkv->nhv", q[:, t], S)
        ym[:, t] = scale * np.einsum("nhk,nhkv->nhv", np.abs(q[:, t]), M)
        Ss.append(S)
        Ms.append(M)
    cut = live[:, :, None, None]
    out = {"y": (y * cut, ym * cut), "s_last": (S, M)}
    if dy is None:
        return out
    R, W = (zero, zero) if ds is None else (ds, np.abs(ds))
    dq, dqm, dk, dkm = np.zeros((4, N, T, H, Dk))
    dv, dvm = np.zeros((2, N, T, H, Dv))
    dl, cross = np.zeros((2, N, T, H))
    for t in range(T - 1, -1, -1):
        qd = scale * q[:, t, :, :, None] * dy[:, t, :, None, :]
        R, W = R + qd, W + np.abs(qd)
        dq[:, t] = scale * np.einsum("nhkv,nhv->nhk", Ss[t + 1], dy[:, t])
        dqm[:, t] = scale * np.einsum("nhkv,nhv->nhk", Ms[t + 1], np.abs(dy[:, t]))
        dk[:, t] = np.einsum("nhkv,nhv->nhk", R, v[:, t])
        dkm[:, t] = np.einsum("nhkv,nhv->nhk", W, np.abs(v[:, t]))
        dv[:, t] = np.einsum("nhkv,nhk->nhv", R, k[:, t])
        dvm[:, t] = np.einsum("nhkv,nhk->nhv", W, np.abs(k[:, t]))
        dl[:, t] = a[:, t] * (Ss[t] * R).sum(axis=(2, 3))
        R, W = a[:, t, :, None, None] * R, a[:, t, :, None, None] * W
        cross[:, t] = (Ms[t] * W).sum(axis=(2, 3))
    # the gates' gradients are formed as the sum of q dq - k dk over the tokens to
    # a border at most SPAN tokens on, and what crosses the border
    per = (np.abs(q) * dqm).sum(axis=3) + (np.abs(k) * dkm).sum(axis=3)
    per = np.concatenate([per, np.zeros((N, SPAN, H))], axis=1)
    total = np.concatenate([np.zeros((N, 1, H)), per.cumsum(axis=1)], axis=1)
    last = (Ms[T] * (0.0 if ds is None else np.abs(ds))).sum(axis=(2, 3))
    dlm = total[:, SPAN:SPAN + T] - total[:, :T] + np.maximum(cross.max(axis=1, initial=0.0), last)[:, None, :]
    slope = 1.0 / (1.0 + np.exp(np.minimum(gate, 700.0))) if form == "logit" else 1.0
    for name, val, mag, heads in (("dq", dq, dqm, Hq), ("dk", dk, dkm, Hk), ("dv", dv, dvm, Hv)):
        out[name] = (gather(val * cut, heads), gather(mag * cut, heads))
    keep = live[:, :, None] & (a > 0)
    out["dgate"] = (np.where(keep, dl * slope, 0.0), np.where(keep, dlm * slope, 0.0))
    out["ds0"] = (R, W)
    return out


def step(q, k, v, gate, form, scale, state):
    """One token: q [N, Hq, Dk], gate [N, H], state [N, H, Dk, Dv] -> (y, its
    magnitude, the new state, its magnitude)."""
    o = attention(q[:, None], k[:, None], v[:, None], gate[:, None], form, scale, s0=state)
    return o["y"][0][:, 0], o["y"][1][:, 0], *o["s_last"]


# ---- block norm ---------------------------------------------------------------

def norm_units(C):
    """Units of 2^-24: a mean over C channels is summed 8 at a time, then over 6
    levels of a wave, then over at most 16 waves; its square root halves the error;
    and some 20 roundings of factors.  The same once more in a gradient."""
    return 2 * (8 + 6 + 16 + C // 512 + 24)


def _norm(v, vm, layer, eps):
    """[..., D] -> n, its magnitude, rho."""
    if layer:
        vm = vm + np.abs(v).mean(-1, keepdims=True)
        v = v - v.mean(-1, keepdims=True)
    rho = 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    # an error d of v moves n by rho (d - n mean(n d)); |n| mean(|n| vm) bounds the second part
    n = v * rho
    return n, rho * (vm + np.abs(n) * (np.abs(n) * vm).mean(-1, keepdims=True)) + np.abs(n), rho


def _norm_grad(n, nm, rho, dn, dnm, layer):
    g = dn - n * (n * dn).mean(-1, keepdims=True)
    m = dnm + np.abs(n) * (nm * np.abs(dn) + np.abs(n) * dnm).mean(-1, keepdims=True) + \
        nm * np.abs((n * dn).mean(-1, keepdims=True))
    if layer:
        g, m = g - dn.mean(-1, keepdims=True), m + dnm.mean(-1, keepdims=True)
    # rho's own error: the norm's, relative
    rel = (np.abs(n) * nm).mean(-1, keepdims=True)
    return g * rho, (m + np.abs(g) * rel) * rho


def block_norm(z, gate=None, x=None, w_post=None, res_scale=None, w_pre=None, groups=0, layer=False, act="silu",
               eps=1e-6, pre=True, dr=None, dy=None):
    """z [R, C] -> dict of (value, magnitude); gradients where dr or dy is given."""
    R, C = z.shape
    one = np.ones(C)
    w1, s, w2 = (one if w is None else w for w in (w_post, res_scale, w_pre))
    p, pm = z, np.abs(z)
    if groups:
        cut = lambda t: t.reshape(R, groups, -1)
        n1, n1m, rho1 = _norm(cut(z), np.abs(cut(z)), layer, eps)
        flat = lambda t: t.reshape(R, C)
        p, pm = flat(n1) * w1, flat(n1m) * np.abs(w1)
    phi = one
    if gate is not None:
        sig = 1.0 / (1.0 + np.exp(-gate))
        phi = gate * sig if act == "silu" else sig
    u, um = p * phi, pm * np.abs(phi)
    r, rm = u * s, um * np.abs(s)
    if x is not None:
        r, rm = x + r, np.abs(x) + rm
    out = {"r": (r, rm)}
    if pre:
        n2, n2m, rho2 = _norm(r, rm, layer, eps)
        out["y"] = (n2 * w2, n2m * np.abs(w2))
    if dr is None and dy is None:
        return out
    d, dm = (np.zeros_like(z), np.zeros_like(z)) if dr is None else (dr, np.abs(dr))
    if dy is not None:
        out["dw_pre"] = ((dy * n2).sum(0), (np.abs(dy) * n2m).sum(0))
        g, gm = _norm_grad(n2, n2m, rho2, dy * w2, np.abs(dy * w2), layer)
        d, dm = d + g, dm + gm
    if x is not None:
        out["dx"] = (d, dm)
    out["dres_scale"] = ((d * u).sum(0), (dm * np.abs(u) + np.abs(d) * um).sum(0))
    du, dum = d * s, dm * np.abs(s)
    if gate is not None:
        rest = 1.0 / (1.0 + np.exp(np.minimum(gate, 700.0)))   # 1 - sig, with its digits
        slope = sig * (1.0 + gate * rest) if act == "silu" else sig * rest
        # (the slope's own terms: sig, gate sig (1 - sig))
        slopem = sig * (1.0 + np.abs(gate) * rest) if act == "silu" else np.abs(slope)
        out["dgate"] = (du * p * slope, (dum * np.abs(p) + np.abs(du) * pm) * slopem)
    dp, dpm = du * phi, dum * np.abs(phi)
    if groups:
        out["dw_post"] = ((dp * flat(n1)).sum(0), (dpm * np.abs(flat(n1)) + np.abs(dp) * flat(n1m)).sum(0))
        g, gm = _norm_grad(n1, n1m, rho1, cut(dp * w1), cut(dpm * np.abs(w1)), layer)
        dp, dpm = flat(g), flat(gm)
    out["dz"] = (dp, dpm)
    return out
