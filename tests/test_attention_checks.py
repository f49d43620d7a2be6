"""What linear attention and the block norms refuse: the C ABI before anything is
launched (placeholder pointers), the binding by the argument's name before a
pointer is taken (CPU tensors); and the oracle's own gradients.  No GPU."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_1906_11367_amd import boxconv as bc

built = pytest.mark.skipif(not os.path.exists(bc.LIB_PATH), reason="libboxconv.so not built")

P = ctypes.c_void_p(0x100000)
P4, P1 = ctypes.c_void_p(0x100004), ctypes.c_void_p(0x100001)
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5, 7


def sizes(**kw):
    d = dict(N=2, T=5, H=6, Hq=2, Hk=3, Hv=6, Dk=8, Dv=4, dt=bc.BC_F32, gate_dt=bc.BC_F32, form=bc.BC_GATE_LOGIT, scale=1.0)
    d.update(kw)
    return bc.bc_attention(**d)


def st(b, r, h):
    return bc.bc_strides(b, r, h)


FWD = dict(q=P, qs=st(80, 16, 8), k=P, ks=st(120, 24, 8), v=P, vs=st(120, 24, 4), gate=P, gs=st(30, 6, 1), s0=P, lengths=P,
           y=P, ys=st(120, 24, 4), s_last=P, states=P, ws=P, ws_bytes=1 << 30, stream=None)
BWD = dict(q=P, qs=st(80, 16, 8), k=P, ks=st(120, 24, 8), v=P, vs=st(120, 24, 4), gate=P, gs=st(30, 6, 1), states=P,
           lengths=P, dy=P, dys=st(120, 24, 4), ds=P, dq=P, dqs=st(80, 16, 8), dk=P, dks=st(120, 24, 8), dv=P,
           dvs=st(120, 24, 4), dgate=P, dgs=st(30, 6, 1), ds0=P, ws=P, ws_bytes=1 << 30, stream=None)
STEP = dict(q=P, qs=st(16, 0, 8), k=P, ks=st(24, 0, 8), v=P, vs=st(24, 0, 4), gate=P, gs=st(6, 0, 1), state=P, state_out=P,
            slots=P, y=P, S=4, stream=None)

# (sizes, status): of every call, and of those with tokens
SIZES = [(dict(N=0), SHAPE), (dict(N=-1), SHAPE), (dict(H=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Hq=4), SHAPE), (dict(Hk=5), SHAPE),
         (dict(Hv=12), SHAPE), (dict(Hv=-1), SHAPE), (dict(Dk=0), SHAPE), (dict(Dv=0), SHAPE), (dict(Dk=129), SHAPE),
         (dict(Dv=129), SHAPE), (dict(N=65536), SHAPE), (dict(dt=bc.BC_I32), DTYPE), (dict(dt=bc.BC_I8), DTYPE),
         (dict(gate_dt=bc.BC_BF16), DTYPE), (dict(gate_dt=7), DTYPE), (dict(form=bc.BC_GATE_VALUE), UNSUPPORTED),
         (dict(form=3), UNSUPPORTED), (dict(form=-1), UNSUPPORTED), (dict(scale=float("nan")), UNSUPPORTED),
         (dict(scale=float("inf")), UNSUPPORTED)]
TOKENS = [(dict(T=0), SHAPE), (dict(T=-5), SHAPE), (dict(T=(1 << 30) + 1), SHAPE), (dict(N=4096, T=1 << 16), SHAPE)]


def call(name, args, bad=None, size=None):
    return getattr(bc.load_library(), name)(size if size is not None else sizes(), *{**args, **(bad or {})}.values())


@built
@pytest.mark.parametrize("name,args,more", [("linear_attention_fwd", FWD, TOKENS), ("linear_attention_bwd", BWD, TOKENS),
                                            ("linear_attention_step", STEP, [])])
def test_sizes_are_refused(name, args, more):
    for bad, status in SIZES + more:
        assert call(name, args, size=sizes(**bad)) == status, bad
        if name != "linear_attention_step" and status == SHAPE:
            assert bc.load_library().bc_linear_attention_workspace_bytes(0, sizes(**bad)) == 0
    assert getattr(bc.load_library(), name)(None, *args.values()) == NULL


@built
@pytest.mark.parametrize("bad,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(gate=None), NULL), (dict(y=None), NULL),
    (dict(q=P4), ALIGN), (dict(k=P4), ALIGN), (dict(v=P4), ALIGN), (dict(gate=P1), ALIGN), (dict(s0=P4), ALIGN),
    (dict(lengths=P4), ALIGN), (dict(y=P4), ALIGN), (dict(s_last=P4), ALIGN), (dict(states=P4), ALIGN),
    (dict(qs=st(-1, 16, 8)), SHAPE), (dict(ks=st(120, -1, 8)), SHAPE), (dict(vs=st(120, 24, -4)), SHAPE),
    (dict(qs=st(1 << 62, 16, 8)), SHAPE), (dict(gs=st(0, -1, 1)), SHAPE), (dict(ys=st(120, 23, 4)), SHAPE),
    (dict(ys=st(119, 24, 4)), SHAPE), (dict(ys=st(120, 24, 3)), SHAPE), (dict(ys=st(0, 24, 4)), SHAPE),
    (dict(ys=st(120, 4, 19)), SHAPE), (dict(ys=st(24, 4, 4)), SHAPE)])
def test_fwd_refuses(bad, status):
    assert call("linear_attention_fwd", FWD, bad) == status


@built
@pytest.mark.parametrize("bad,status", [
    (dict(q=None), NULL), (dict(gate=None), NULL), (dict(states=None), NULL), (dict(dy=None), NULL), (dict(dq=None), NULL),
    (dict(dk=None), NULL), (dict(dv=None), NULL), (dict(states=P4), ALIGN), (dict(dy=P4), ALIGN), (dict(dq=P4), ALIGN),
    (dict(dk=P4), ALIGN), (dict(dv=P4), ALIGN), (dict(dgate=P1), ALIGN), (dict(ds=P4), ALIGN), (dict(ds0=P4), ALIGN),
    (dict(lengths=P4), ALIGN), (dict(dys=st(-1, 24, 4)), SHAPE), (dict(dqs=st(80, 15, 8)), SHAPE),
    (dict(dks=st(120, 24, 7)), SHAPE), (dict(dvs=st(0, 0, 0)), SHAPE), (dict(dgs=st(30, 5, 1)), SHAPE),
    (dict(dgs=st(0, 0, 1)), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws_bytes=16), WORKSPACE), (dict(ws=P4), ALIGN)])
def test_bwd_refuses(bad, status):
    assert call("linear_attention_bwd", BWD, bad) == status


@built
def test_fwd_workspace():
    big = sizes(N=1, T=100000)
    args = dict(FWD, qs=st(0, 16, 8), ks=st(0, 24, 8), vs=st(0, 24, 4), gs=st(0, 6, 1), ys=st(0, 24, 4))
    need = bc.load_library().bc_linear_attention_workspace_bytes(0, big)
    assert need > 0
    for bad, status in ((dict(ws=None), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE), (dict(ws=P4), ALIGN)):
        assert call("linear_attention_fwd", args, bad, big) == status


@built
@pytest.mark.parametrize("bad,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(gate=None), NULL), (dict(state=None), NULL),
    (dict(state_out=None), NULL), (dict(y=None), NULL), (dict(S=0), SHAPE), (dict(S=-1), SHAPE), (dict(slots=None, S=1), SHAPE),
    (dict(qs=st(-1, 0, 8)), SHAPE), (dict(q=P4), ALIGN), (dict(gate=P1), ALIGN), (dict(state=P4), ALIGN),
    (dict(state_out=P4), ALIGN), (dict(slots=P4), ALIGN), (dict(y=P4), ALIGN)])
def test_step_refuses(bad, status):
    assert call("linear_attention_step", STEP, bad) == status


@built
def test_attention_queries():
    lib = bc.load_library()
    assert lib.bc_linear_attention_workspace_bytes(2, sizes()) == 0
    assert lib.bc_linear_attention_workspace_bytes(0, None) == 0
    assert lib.bc_linear_attention_states_bytes(2, 0, 3, 8, 8) == 0
    assert lib.bc_linear_attention_states_bytes(2, 5, 3, 8, 129) == 0
    assert lib.bc_linear_attention_states_bytes(2, 5, 3, 8, 4) == 2 * 3 * 8 * 4 * 4 * 2


NORM = dict(R=3, C=24, groups=3, kind=0, act=0, dt=bc.BC_F32, eps=1e-6)
NFWD = dict(z=P, zs=24, gate=P, gs=24, x=P, xs=24, w1=P, s=P, w2=P, r=P, rs=24, y=P, ys=24, stream=None)
NBWD = dict(z=P, zs=24, gate=P, gs=24, x=P, xs=24, w1=P, s=P, w2=P, dr=P, drs=24, dy=P, dys=24, dz=P, dzs=24, dgate=P, dgs=24,
            dx=P, dxs=24, dw1=P, dsc=P, dw2=P, ws=P, ws_bytes=1 << 20, stream=None)


def norm(name, args, bad=None, **size):
    return getattr(bc.load_library(), name)(bc.bc_norm(**{**NORM, **size}), *{**args, **(bad or {})}.values())


@built
@pytest.mark.parametrize("name,args", [("block_norm_fwd", NFWD), ("block_norm_bwd", NBWD)])
@pytest.mark.parametrize("bad,status", [
    (dict(R=0), SHAPE), (dict(C=0), SHAPE), (dict(C=16385, groups=1), SHAPE), (dict(groups=-1), SHAPE), (dict(groups=5), SHAPE),
    (dict(groups=48), SHAPE), (dict(C=8192, groups=8192), SHAPE), (dict(dt=bc.BC_I32), DTYPE), (dict(dt=9), DTYPE),
    (dict(kind=2), UNSUPPORTED), (dict(act=-1), UNSUPPORTED), (dict(eps=0.0), UNSUPPORTED), (dict(eps=-1.0), UNSUPPORTED),
    (dict(eps=float("nan")), UNSUPPORTED), (dict(eps=1e-40), UNSUPPORTED), (dict(eps=float("inf")), UNSUPPORTED)])
def test_norm_sizes_are_refused(name, args, bad, status):
    assert norm(name, args, **bad) == status


@built
@pytest.mark.parametrize("bad,status", [
    (dict(z=None), NULL), (dict(r=None, y=None), NULL), (dict(y=None), UNSUPPORTED), (dict(zs=23), SHAPE), (dict(gs=0), SHAPE),
    (dict(xs=-24), SHAPE), (dict(rs=23), SHAPE), (dict(ys=1 << 40), SHAPE), (dict(z=P4), ALIGN), (dict(gate=P4), ALIGN),
    (dict(x=P4), ALIGN), (dict(w1=P4), ALIGN), (dict(s=P4), ALIGN), (dict(w2=P4), ALIGN), (dict(r=P4), ALIGN),
    (dict(y=P4), ALIGN)])
def test_norm_fwd_refuses(bad, status):
    assert norm("block_norm_fwd", NFWD, bad) == status


@built
def test_norm_weights_without_their_norm_are_refused():
    assert norm("block_norm_fwd", NFWD, groups=0) == UNSUPPORTED
    assert norm("block_norm_bwd", NBWD, dict(w1=None), groups=0) == UNSUPPORTED
    assert norm("block_norm_bwd", NBWD, dict(dy=None)) == UNSUPPORTED


@built
@pytest.mark.parametrize("bad,status", [
    (dict(z=None), NULL), (dict(dr=None, dy=None), NULL), (dict(gate=None), NULL), (dict(x=None), NULL), (dict(drs=23), SHAPE),
    (dict(dzs=0), SHAPE), (dict(dgs=23), SHAPE), (dict(dxs=23), SHAPE), (dict(dr=P4), ALIGN), (dict(dz=P4), ALIGN),
    (dict(dgate=P4), ALIGN), (dict(dx=P4), ALIGN), (dict(dw1=P4), ALIGN), (dict(dsc=P4), ALIGN), (dict(dw2=P4), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=8), WORKSPACE), (dict(ws=P4), ALIGN)])
def test_norm_bwd_refuses(bad, status):
    assert norm("block_norm_bwd", NBWD, bad) == status


# ---- the binding --------------------------------------------------------------

bf16, f64, i32 = torch.bfloat16, torch.float64, torch.int32


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


STATES = 2 * 6 * 8 * 4 * 2
CALLS = {
    "linear_attention_fwd": dict(q=t(2, 5, 2, 8), k=t(2, 5, 3, 8), v=t(2, 5, 6, 4), gate=t(2, 5, 6), y=t(2, 5, 6, 4),
                                 s0=t(2, 6, 8, 4), s_last=t(2, 6, 8, 4), lengths=t(2, dtype=i32), states=t(STATES)),
    "linear_attention_bwd": dict(q=t(2, 5, 2, 8), k=t(2, 5, 3, 8), v=t(2, 5, 6, 4), gate=t(2, 5, 6), states=t(STATES),
                                 grad_y=t(2, 5, 6, 4), grad_q=t(2, 5, 2, 8), grad_k=t(2, 5, 3, 8), grad_v=t(2, 5, 6, 4),
                                 grad_gate=t(2, 5, 6), grad_s_last=t(2, 6, 8, 4), grad_s0=t(2, 6, 8, 4),
                                 lengths=t(2, dtype=i32)),
    "linear_attention_step": dict(q=t(2, 2, 8), k=t(2, 3, 8), v=t(2, 6, 4), gate=t(2, 6), state=t(4, 6, 8, 4),
                                  y=t(2, 6, 4), slots=t(2, dtype=i32), state_out=t(4, 6, 8, 4)),
    "block_norm_fwd": dict(z=t(5, 24), gate=t(5, 24), x=t(5, 24), w_post=t(24), res_scale=t(24), w_pre=t(24), r=t(5, 24),
                           y=t(5, 24), groups=3),
    "block_norm_bwd": dict(z=t(5, 24), gate=t(5, 24), x=t(5, 24), w_post=t(24), res_scale=t(24), w_pre=t(24),
                           grad_r=t(5, 24), grad_y=t(5, 24), grad_z=t(5, 24), grad_gate=t(5, 24), grad_x=t(5, 24),
                           grad_w_post=t(24), grad_res_scale=t(24), grad_w_pre=t(24), groups=3),
}
LA, LB, LS, NF, NB = CALLS


@built
@pytest.mark.parametrize("call", CALLS)
def test_a_call_without_a_fault_asks_for_the_gpu(call):
    with pytest.raises(bc.BoxConvError, match="must be on the GPU"):
        getattr(bc, call)(**CALLS[call])


@built
@pytest.mark.parametrize("call,bad,says", [
    (LA, dict(q=t(2, 5, 16)), "q must be"), (LA, dict(q=None), "q must be"), (LA, dict(q=t(2, 5, 2, 8, dtype=f64)), "q must be"),
    (LA, dict(q=t(2, 5, 2, 8, dtype=bf16)), "q has dtype"), (LA, dict(q=t(2, 4, 2, 8)), "q has shape"),
    (LA, dict(k=t(2, 5, 3, 7)), "k has shape"), (LA, dict(k=t(2, 5, 4, 8)), "k has 4 heads"), (LA, dict(v=t(2, 5, 6, 5)), "v has shape"),
    (LA, dict(v=t(2, 5, 0, 4)), "v has 0 heads"), (LA, dict(gate=t(2, 5, 5)), "gate has shape"), (LA, dict(gate=t(5)), "gate has shape"),
    (LA, dict(gate=t(2, 5, 6, dtype=bf16)), "gate must be"), (LA, dict(gate=None), "gate must be"), (LA, dict(y=None), "y must be"),
    (LA, dict(y=t(2, 5, 4, 6).transpose(2, 3)), "y must be contiguous"),
    (LA, dict(k=t(2, 5, 8, 3).transpose(2, 3)), "k must be contiguous"), (LA, dict(s0=t(2, 6, 4, 8)), "s0 has shape"),
    (LA, dict(s_last=t(2, 6, 8, 4, dtype=bf16)), "s_last has dtype"), (LA, dict(lengths=t(2)), "lengths has dtype"),
    (LA, dict(lengths=t(3, dtype=i32)), "lengths has shape"), (LA, dict(states=t(STATES - 1)), "states has"),
    (LB, dict(grad_y=None), "grad_y must be"), (LB, dict(grad_y=t(2, 5, 6, 4, dtype=bf16)), "has dtype"),
    (LB, dict(grad_q=t(2, 5, 6, 8)), "grad_q has shape"), (LB, dict(grad_k=None), "grad_k must be"),
    (LB, dict(grad_v=t(2, 5, 6, 4, dtype=bf16)), "grad_v has dtype"), (LB, dict(grad_gate=t(6)), "grad_gate has shape"),
    (LB, dict(grad_gate=t(2, 5, 6, dtype=bf16)), "grad_gate has dtype"), (LB, dict(states=None), "states must be"),
    (LB, dict(states=t(3)), "states has"), (LB, dict(grad_s_last=t(2, 6, 8)), "grad_s_last has shape"),
    (LB, dict(grad_s0=t(1, 6, 8, 4)), "grad_s0 has shape"),
    (LS, dict(q=t(2, 1, 2, 8)), "q must be"), (LS, dict(state=t(4, 6, 8)), "state must be"), (LS, dict(state=t(4, 6, 4, 8)), "state has shape"),
    (LS, dict(state=None), "state must be"), (LS, dict(state_out=t(3, 6, 8, 4)), "state_out has shape"),
    (LS, dict(slots=t(2)), "slots has dtype"), (LS, dict(gate=t(2, 5)), "gate has shape"),
    (NF, dict(z=t(24)), "z must be"), (NF, dict(z=None), "z must be"), (NF, dict(z=t(5, 24, dtype=f64)), "z must be"),
    (NF, dict(gate=t(5, 23)), "gate has shape"), (NF, dict(x=t(5, 24, dtype=bf16)), "x has dtype"), (NF, dict(w_post=t(8)), "w_post has shape"),
    (NF, dict(res_scale=t(24, dtype=bf16)), "res_scale has dtype"), (NF, dict(w_pre=t(1, 24)), "w_pre has shape"),
    (NF, dict(r=t(4, 24)), "r has shape"), (NF, dict(y=t(24, 5).t()), "y must be contiguous"),
    (NB, dict(grad_r=t(5, 25)), "grad_r has shape"), (NB, dict(grad_y=t(5, 24, dtype=bf16)), "grad_y has dtype"),
    (NB, dict(grad_z=t(5, 24, 1)), "grad_z has shape"), (NB, dict(grad_w_post=t(5, 24)), "grad_w_post has shape"),
    (NB, dict(grad_w_pre=t(24, dtype=f64)), "grad_w_pre has dtype")])
def test_the_binding_names_what_it_refuses(call, bad, says):
    with pytest.raises(bc.BoxConvError, match=says):
        getattr(bc, call)(**{**CALLS[call], **bad})


@built
def test_rows_that_are_not_equally_far_apart():
    z = t(4, 9, 64)[:, :5, :32]
    with pytest.raises(bc.BoxConvError, match="equally far apart"):
        bc.block_norm_fwd(z, y=t(4, 5, 32))


# ---- the oracles --------------------------------------------------------------

@pytest.mark.parametrize("form", ["logit", "log"])
@pytest.mark.parametrize("lengths", [None, [7, 0, 3]])
def test_attention_oracles_gradients_are_the_losss_differences(form, lengths):
    rng = np.random.default_rng(1)
    N, T, H, Dk, Dv = 3, 7, 4, 3, 2
    shapes = dict(q=(N, T, 2, Dk), k=(N, T, 1, Dk), v=(N, T, 4, Dv), gate=(N, T, H), s0=(N, H, Dk, Dv))
    at = {n: rng.standard_normal(s) for n, s in shapes.items()}
    dy, ds = rng.standard_normal((N, T, H, Dv)), rng.standard_normal((N, H, Dk, Dv))

    def loss(d):
        o = A.attention(d["q"], d["k"], d["v"], d["gate"], form, 0.7, d["s0"], lengths)
        return (o["y"][0] * dy).sum() + (o["s_last"][0] * ds).sum()

    g = A.attention(at["q"], at["k"], at["v"], at["gate"], form, 0.7, at["s0"], lengths, dy, ds)
    for name, shape in shapes.items():
        w, eps = rng.standard_normal(shape), 1e-5
        diff = (loss({**at, name: at[name] + eps * w}) - loss({**at, name: at[name] - eps * w})) / (2 * eps)
        assert abs(diff - (g["d" + name][0] * w).sum()) < 1e-6, name


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("groups,act,x,pre", [(0, "", False, True), (3, "silu", True, True), (1, "sigmoid", False, False),
                                              (4, "silu", False, True), (1, "", True, True)])
def test_norm_oracles_gradients_are_the_losss_differences(layer, groups, act, x, pre):
    rng = np.random.default_rng(2)
    R, C = 4, 12
    new = lambda on, *s: rng.standard_normal(s) if on else None
    at = dict(z=new(True, R, C), gate=new(act, R, C), x=new(x, R, C), w_post=new(groups, C), res_scale=new(True, C), w_pre=new(pre, C))
    dr, dy = new(True, R, C), new(pre, R, C)
    how = dict(groups=groups, layer=layer, act=act, eps=1e-3, pre=pre)

    def loss(d):
        o = A.block_norm(**d, **how)
        return (o["r"][0] * dr).sum() + ((o["y"][0] * dy).sum() if pre else 0.0)

    g = A.block_norm(**at, **how, dr=dr, dy=dy)
    for name, v in at.items():
        if v is None:
            continue
        w, eps = rng.standard_normal(v.shape), 1e-5
        diff = (loss({**at, name: v + eps * w}) - loss({**at, name: v - eps * w})) / (2 * eps)
        assert abs(diff - (g["d" + name][0] * w).sum()) < 1e-6, name


def test_oracles_hold_by_hand():
    one = np.ones((1, 2, 1, 1))
    o = A.attention(2 * one, 3 * one, 5 * one, np.full((1, 2, 1), np.log(0.5)), "log", 1.0)
    assert np.allclose(o["y"][0].ravel(), [30, 45]) and np.allclose(o["s_last"][0], 22.5)
    n = A.block_norm(np.array([[3.0, 4.0]]), eps=0.0)["y"][0]
    assert np.allclose(n, np.array([[3, 4]]) / np.sqrt(12.5))
    n = A.block_norm(np.array([[3.0, 5.0]]), layer=True, eps=0.0)["y"][0]
    assert np.allclose(n, [[-1, 1]])


def test_sizes_of_2_31_are_refused():
    """(A size that the library's 32 bits cannot hold; the tensors are one element seen often.)"""
    one = torch.zeros(1)
    many = one.expand(2 ** 31, 8)
    with pytest.raises(bc.BoxConvError, match="2\\^31"):
        bc.block_norm_fwd(many, r=many)
    with pytest.raises(bc.BoxConvError, match="2\\^31"):
        bc.block_norm_bwd(many, grad_r=many, grad_z=many)
    t = one.expand(2 ** 31, 1, 8)
    with pytest.raises(bc.BoxConvError, match="2\\^31"):
        bc.linear_attention_step(t, t, t, one.expand(2 ** 31, 1), one.expand(1, 1, 8, 8), t)
    t = one.expand(1, 2 ** 31, 1, 8)
    with pytest.raises(bc.BoxConvError, match="2\\^31"):
        bc.linear_attention_fwd(t, t, t, one.expand(1, 2 ** 31, 1), t)


def test_arguments_that_are_no_tensors_are_refused():
    t, g, s = torch.zeros(1, 1, 8), torch.zeros(1, 1), torch.zeros(1, 1, 8, 8)
    for bad in (None, 3.0, [1.0], t.numpy(), t.to_sparse()):
        with pytest.raises((bc.BoxConvError, RuntimeError)):
            bc.linear_attention_step(bad, t, t, g, s, t)
        with pytest.raises((bc.BoxConvError, RuntimeError)):
            bc.linear_attention_fwd(t[None], bad, t[None], g[None], t[None])
        with pytest.raises((bc.BoxConvError, RuntimeError)):
            bc.block_norm_fwd(bad, r=t)


# ---- the server's pool ---------------------------------------------------------

def test_a_pool_that_is_set_stays_where_it_is():
    """A graph captured before has its address; prefill's extra row stays behind it."""
    from paper_1906_11367_amd.attention import LinearAttentionServer
    server = object.__new__(LinearAttentionServer)
    server.state = torch.zeros((3, 2, 4, 4))
    at, new = server.state.data_ptr(), torch.randn(3, 2, 4, 4)
    for value, want in ((new, new), (new.double(), new), (new[[2, 0, 1]], new[[2, 0, 1]])):
        server.state = value
        assert server.state.data_ptr() == at and torch.equal(server.state, want)
    server.state = server.state.transpose(2, 3)   # a view of itself
    assert server.state.data_ptr() == at and torch.equal(server.state, new[[2, 0, 1]].transpose(2, 3))
    server.state = torch.ones(5, 2, 4, 4)         # another number of slots
    assert server.state.shape == (5, 2, 4, 4) and (server.state == 1).all()
    assert server._rows.shape[0] == 6 and (server._rows[-1] == 0).all()
    for bad in (torch.ones(5, 2, 4, 5), torch.ones(3, 2, 4)):
        with pytest.raises(ValueError, match="state must be"):
            server.state = bad
    assert (server.state == 1).all()


@built
@pytest.mark.parametrize("name", ["w_in", "w_out"])
def test_a_plans_matrices_have_their_shapes(name):
    """The other way round they have as many elements."""
    from paper_1906_11367_amd.attention import LinearAttentionPlan
    plan = LinearAttentionPlan(1, 4, 24, 2, 8, 8, device="cpu")
    W = plan.shape.width
    w = {"w_pre": t(24), "w_in": t(24, W), "w_head": t(16), "w_out": t(16, 24), "w_post": t(24), "res_scale": t(24)}
    w[name] = t(*w[name].shape[::-1])
    with pytest.raises(bc.BoxConvError, match=f"{name} has shape"):
        plan.forward(t(1, 4, 24), w)
    with pytest.raises(bc.BoxConvError, match=f"{name} has shape"):
        plan.backward(t(1, 4, 24), w, t(1, 4, 24))
