"""The recurrent layer's operators in 64 bits, step by step (NumPy).

Shares no code with the library.  Sequences are handled time first, [T, N, C];
`seq` and `unseq` turn a layout's order into that and back.  Beside each
forward and gradient value a bound on the error of a 32-bit evaluation is
formed by the same recurrence: every step's coefficients and roundings
contribute k units of 2^-24 of the magnitudes that meet there, carried on by
the coefficients' absolute values.
"""
import numpy as np

EPS = 2.0 ** -24     # unit roundoff of fp32
U_BF16 = 2.0 ** -8   # unit roundoff of bf16


def seq(v, layout):
    """[N, T, C] ("tokens") or [N, C, T] ("maps") -> [T, N, C], fp64."""
    return np.ascontiguousarray(np.asarray(v, np.float64).transpose((1, 0, 2) if layout == "tokens" else (2, 0, 1)))


def unseq(v, layout):
    return np.ascontiguousarray(v.transpose((1, 0, 2) if layout == "tokens" else (1, 2, 0)))


def coefficients(gate, form):
    """a and the input's coefficient c."""
    if form == "value":
        return gate, np.ones_like(gate)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))


def _live(lengths, T, N):
    if lengths is None:
        return np.ones((T, N, 1), bool)
    n = np.clip(np.asarray(lengths, np.int64), 0, T)
    return (np.arange(T)[:, None] < n[None, :])[:, :, None]


def _units(gate, form, base=8.0):
    """Units of 2^-24 by which a step's coefficients and its own arithmetic may
    be off: a few roundings, and for the logit form |gate| more (the argument
    of the exponential is a rounded product)."""
    if form == "value":
        return np.full_like(gate, base)
    return base + np.minimum(np.abs(np.where(np.isfinite(gate), gate, 0.0)), 100.0)


def scan_forward(gate, x, h0=None, lengths=None, form="logit"):
    """[T, N, C] -> (h [T + 1, N, C] with h[0] = h0, y, bound of h)."""
    T, N, C = gate.shape
    live = _live(lengths, T, N)
    gate, x = np.where(live, gate, 0.0), np.where(live, x, 0.0)
    a, c = coefficients(gate, form)
    k = _units(gate, form) * EPS
    h = np.zeros((T + 1, N, C))
    e = np.zeros((T + 1, N, C))
    m = np.zeros((N, C))
    if h0 is not None:
        h[0] = h0
        m = np.abs(h[0])
    for t in range(T):
        on = live[t]
        h[t + 1] = np.where(on, a[t] * h[t] + c[t] * x[t], h[t])
        parts = np.abs(a[t]) * m + np.abs(c[t] * x[t])
        e[t + 1] = np.where(on, np.abs(a[t]) * e[t] + k[t] * parts, e[t])
        m = np.where(on, parts, m)
    return h, np.where(live, h[1:], 0.0), e + 1e-36


def scan_backward(gate, x, gy, h0=None, gh_last=None, lengths=None, form="logit"):
    """-> dict of gradients and of their bounds ([T, N, C], and [N, C] for h0)."""
    T, N, C = gate.shape
    live = _live(lengths, T, N)
    h, _, eh = scan_forward(gate, x, h0, lengths, form)
    gate, x, gy = (np.where(live, v, 0.0) for v in (gate, x, gy))
    a, c = coefficients(gate, form)
    k = _units(gate, form) * EPS
    r = np.zeros((N, C)) if gh_last is None else np.array(gh_last, np.float64)
    er, m = np.zeros((N, C)), np.abs(r)
    out = {n: np.zeros((T, N, C)) for n in ("gate", "x", "gate_bound", "x_bound")}
    for t in range(T - 1, -1, -1):
        on = live[t]
        delta, size = gy[t] + r, np.abs(gy[t]) + m
        ed = er + k[t] * size
        if form == "value":
            gx, ex = delta, ed
            gg, eg = delta * h[t], ed * np.abs(h[t]) + size * eh[t] + k[t] * np.abs(delta * h[t])
        else:
            gx, ex = delta * c[t], ed * c[t] + k[t] * np.abs(delta * c[t])
            w, d = a[t] * c[t], h[t] - x[t]
            gg = delta * d * w
            eg = (ed * np.abs(d) + size * (eh[t] + EPS * (np.abs(h[t]) + np.abs(x[t])))) * w + 2 * k[t] * np.abs(gg)
        for name, v in (("gate", gg), ("x", gx), ("gate_bound", eg), ("x_bound", ex)):
            out[name][t] = np.where(on, v, 0.0)
        r = np.where(on, a[t] * delta, r)
        er = np.where(on, np.abs(a[t]) * ed + k[t] * np.abs(a[t]) * size, er)
        m = np.where(on, np.abs(a[t]) * size, m)
    out["h0"], out["h0_bound"] = r, er + 1e-36
    for name in ("gate_bound", "x_bound"):
        out[name] += 1e-36
    return out


def codes(v):
    """8-bit codes (whole numbers in fp64) and fp32 scales of the rows of v, by
    the definition: 32-bit arithmetic, codes to nearest even."""
    v = np.asarray(v, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(v).max(axis=1, keepdims=True)
        bad = ~np.isfinite(v).all(axis=1, keepdims=True)
        live = ~bad & (top >= np.float32(2.0 ** -100))
        safe = np.where(live, top, np.float32(1))
        inv = (np.float32(127) / safe).astype(np.float32)
        q = np.where(live, np.rint(np.where(live, v, np.float32(0)) * inv), 0.0).astype(np.float64)
        scale = np.where(bad, np.float32(np.nan), np.where(live, safe / np.float32(127), np.float32(0)))
    return q, scale.astype(np.float32)[:, 0]


def mix_codes(q, scale, wq, wscale, bias=None, relu=False):
    """[rows, K] codes by [M, K] codes -> [rows, M], and a bound on the error of
    the four 32-bit roundings after the exact product."""
    s, w = np.asarray(scale, np.float64)[:, None], np.asarray(wscale, np.float64)[None, :]
    z = (np.asarray(q, np.float64) @ np.asarray(wq, np.float64).T) * s * w
    bound = 4 * EPS * np.abs(z)
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
        bound = bound + 2 * EPS * np.abs(z)
    return (np.maximum(z, 0.0) if relu else z), bound + 1e-36
