"""What the recurrent layer's entry points refuse: the C ABI before anything is
launched (placeholder pointers), the binding before a pointer is taken (CPU
tensors).  No GPU."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import recurrent_oracle as R
from paper_1906_11367_amd import boxconv as bc

pytestmark = pytest.mark.skipif(not os.path.exists(bc.LIB_PATH), reason="libboxconv.so not built")

P16 = ctypes.c_void_p(0x100000)
P4 = ctypes.c_void_p(0x100004)
E = bc.BoxConvError
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5, 7


def changed(args, **kw):
    return list({**args, **kw}.values())


FWD = dict(gate=P16, x=P16, dt=bc.BC_F32, bs=5 * 8, rs=8, h0=P16, lengths=P16, y=P16, y_dt=bc.BC_F32, h_last=P16,
           states=P16, N=2, T=5, C=8, form=0, layout=0, ws=None, ws_bytes=0, stream=None)
BWD = dict(gate=P16, x=P16, dt=bc.BC_F32, bs=5 * 8, rs=8, states=P16, lengths=P16, gy=P16, gh=P16, gg=P16, gx=P16,
           out_dt=bc.BC_F32, gbs=5 * 8, grs=8, gh0=P16, N=2, T=5, C=8, form=0, layout=0, ws=None, ws_bytes=0,
           stream=None)
STEP = dict(gate=P16, x=P16, dt=bc.BC_F32, rs=8, state=P16, state_out=P16, slots=P16, y=P16, N=2, C=8, S=4, form=0,
            stream=None)
QUANT = dict(src=P16, dt=bc.BC_F32, bs=40, rs=8, q=P16, scale=P16, N=2, K=8, P=5, layout=0, stream=None)
MIX = dict(wq=P16, ws=P16, x=P16, x_dt=bc.BC_F32, bs=40, rs=8, x_scale=None, bias=P16, out=P16, out_dt=bc.BC_F32, N=2,
           M=3, K=8, P=5, relu=0, layout=0, wsp=P16, wsp_bytes=1 << 20, stream=None)

COMMON = [(dict(gate=None), NULL), (dict(x=None), NULL), (dict(N=0), SHAPE), (dict(T=0), SHAPE), (dict(C=0), SHAPE),
          (dict(N=-1), SHAPE), (dict(T=(1 << 30) + 1), SHAPE), (dict(C=65537, rs=65537, bs=1 << 40), SHAPE),
          (dict(N=65536, C=1024, rs=1024, bs=1 << 30, layout=1), SHAPE),
          (dict(N=65536, T=1 << 24, C=64, rs=64, bs=1 << 40), SHAPE), (dict(rs=7), SHAPE), (dict(bs=39), SHAPE),
          (dict(rs=-8), SHAPE), (dict(bs=-40), SHAPE), (dict(bs=1 << 62), SHAPE), (dict(rs=1 << 62), SHAPE),
          (dict(dt=bc.BC_I32), DTYPE), (dict(dt=bc.BC_I8), DTYPE), (dict(dt=9), DTYPE), (dict(form=2), UNSUPPORTED),
          (dict(form=-1), UNSUPPORTED), (dict(layout=2), UNSUPPORTED), (dict(gate=P4), ALIGN), (dict(x=P4), ALIGN),
          (dict(lengths=P4), ALIGN), (dict(states=P4), ALIGN)]


@pytest.mark.parametrize("bad,status", COMMON + [
    (dict(y=None), NULL), (dict(y=P4), ALIGN), (dict(h0=P4), ALIGN), (dict(h_last=P4), ALIGN),
    (dict(y_dt=bc.BC_I32), DTYPE), (dict(dt=bc.BC_BF16), DTYPE),            # bf16 in, fp32 out
    (dict(layout=1, rs=4, bs=40), SHAPE)])                                   # maps: rows of T
def test_scan_fwd_refuses(bad, status):
    assert bc.load_library().gated_scan_fwd(*changed(FWD, **bad)) == status


@pytest.mark.parametrize("bad,status", COMMON + [
    (dict(gy=None), NULL), (dict(gg=None), NULL), (dict(gx=None), NULL), (dict(states=None), NULL),
    (dict(gy=P4), ALIGN), (dict(gg=P4), ALIGN), (dict(gx=P4), ALIGN), (dict(gh=P4), ALIGN), (dict(gh0=P4), ALIGN),
    (dict(grs=7), SHAPE), (dict(gbs=39), SHAPE), (dict(out_dt=bc.BC_I8), DTYPE), (dict(dt=bc.BC_BF16), DTYPE)])
def test_scan_bwd_refuses(bad, status):
    assert bc.load_library().gated_scan_bwd(*changed(BWD, **bad)) == status


@pytest.mark.parametrize("bad,status", [
    (dict(gate=None), NULL), (dict(x=None), NULL), (dict(state=None), NULL), (dict(state_out=None), NULL),
    (dict(y=None), NULL), (dict(N=0), SHAPE), (dict(C=0), SHAPE), (dict(S=0), SHAPE), (dict(C=65537, rs=65537), SHAPE),
    (dict(N=(1 << 20) + 1), SHAPE), (dict(N=65536, C=65536, rs=65536), SHAPE), (dict(slots=None, N=5), SHAPE), (dict(rs=7), SHAPE), (dict(dt=bc.BC_I32), DTYPE),
    (dict(form=5), UNSUPPORTED), (dict(gate=P4), ALIGN), (dict(state=P4), ALIGN), (dict(state_out=P4), ALIGN),
    (dict(slots=P4), ALIGN), (dict(y=P4), ALIGN)])
def test_scan_step_refuses(bad, status):
    assert bc.load_library().gated_scan_step(*changed(STEP, **bad)) == status


@pytest.mark.parametrize("bad,status", [
    (dict(src=None), NULL), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(N=0), SHAPE), (dict(K=0), SHAPE),
    (dict(P=0), SHAPE), (dict(K=65537, rs=65537, bs=1 << 30), SHAPE), (dict(N=65536, P=65536, bs=1 << 20), SHAPE),
    (dict(rs=7), SHAPE), (dict(bs=39), SHAPE), (dict(layout=1, rs=4), SHAPE), (dict(layout=3), UNSUPPORTED),
    (dict(dt=bc.BC_I8), DTYPE), (dict(src=P4), ALIGN), (dict(q=P4), ALIGN), (dict(scale=P4), ALIGN)])
def test_quantize_refuses(bad, status):
    assert bc.load_library().quantize_i8(*changed(QUANT, **bad)) == status


@pytest.mark.parametrize("bad,status", [
    (dict(wq=None), NULL), (dict(ws=None), NULL), (dict(x=None), NULL), (dict(out=None), NULL),
    (dict(x_dt=bc.BC_I8), NULL),                                             # codes without scales
    (dict(x_scale=P16), UNSUPPORTED), (dict(layout=-1), UNSUPPORTED), (dict(N=0), SHAPE), (dict(M=0), SHAPE),
    (dict(K=0), SHAPE), (dict(P=0), SHAPE), (dict(M=65537), SHAPE), (dict(K=65537), SHAPE),
    (dict(N=1024, P=1 << 20, M=65536), SHAPE), (dict(rs=7), SHAPE), (dict(bs=39), SHAPE),
    (dict(x_dt=bc.BC_I32), DTYPE), (dict(out_dt=bc.BC_I8), DTYPE), (dict(wq=P4), ALIGN), (dict(ws=P4), ALIGN),
    (dict(x=P4), ALIGN), (dict(out=P4), ALIGN), (dict(bias=P4), ALIGN), (dict(wsp=None), WORKSPACE),
    (dict(wsp_bytes=16), WORKSPACE), (dict(wsp=P4), ALIGN)])
def test_mix_i8_refuses(bad, status):
    args = dict(MIX, M=300, P=200, bs=200 * 8) if "wsp" in str(bad) else MIX
    assert bc.load_library().pointwise_mix_i8(*changed(args, **bad)) == status


def test_sizes():
    lib = bc.load_library()
    assert [lib.bc_i8_pitch(k) for k in (0, -1, 1, 128, 129, 65536, 65537)] == [0, 0, 128, 128, 256, 65536, 0]
    assert lib.bc_gated_scan_states_bytes(2, 5, 8, 2) == 0
    assert lib.bc_gated_scan_states_bytes(0, 5, 8, 0) == 0
    assert lib.bc_gated_scan_states_bytes(2, 5, 8, 0) >= 2 * 8 * 4
    for bad in ((2, 2, 5, 8, 1, 0), (0, 0, 5, 8, 1, 0), (0, 2, 5, 8, 0, 0), (0, 2, 5, 8, 1, 7)):
        assert lib.bc_gated_scan_workspace_bytes(*bad) == 0
    assert lib.bc_mix_i8_workspace_bytes(1, 300, 500, 200, bc.BC_I8, 0) == 0
    assert lib.bc_mix_i8_workspace_bytes(1, 300, 500, 200, bc.BC_I32, 0) == 0
    assert lib.bc_mix_i8_workspace_bytes(1, 300, 500, 200, bc.BC_F32, 9) == 0
    assert lib.bc_mix_i8_workspace_bytes(1, 300, 500, 2000, bc.BC_F32, 0) >= 2000 * (512 + 4)


def test_a_longer_scans_workspace_serves_shorter_ones():
    lib = bc.load_library()
    for op in (0, 1):
        for dt in (bc.BC_F32, bc.BC_BF16):
            sizes = [lib.bc_gated_scan_workspace_bytes(op, 1, T, 200, dt, bc.BC_TOKENS)
                     for T in (1, 128, 129, 257, 300, 2048, 16256, 16257, 16384, 16385, 40000, 300000)]
            assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[-1] > 0


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


bf16, f64 = torch.bfloat16, torch.float64


@pytest.mark.parametrize("bad", [
    dict(gate=t(2, 5, 7)), dict(gate=t(2, 5, 8, dtype=bf16)), dict(gate=None), dict(x=t(2, 40)), dict(x=None),
    dict(x=t(2, 5, 8, dtype=f64)), dict(y=t(2, 5, 9)), dict(y=t(2, 5, 8, dtype=f64)), dict(h0=t(2, 7)),
    dict(h_last=t(2, 8, dtype=bf16)), dict(lengths=t(2)), dict(lengths=t(3, dtype=torch.int32)), dict(states=t(3)),
    dict(layout=4)])
def test_scan_fwd_binding_refuses(bad):
    a = dict(gate=t(2, 5, 8), x=t(2, 5, 8), y=t(2, 5, 8))
    a.update(bad)
    with pytest.raises(E):
        bc.gated_scan_fwd(**a)


@pytest.mark.parametrize("bad", [
    dict(gate=t(2, 5, 7)), dict(grad_y=t(2, 5, 9)), dict(grad_y=t(2, 5, 8, dtype=bf16)), dict(grad_y=None),
    dict(states=t(3)), dict(states=None), dict(grad_x=t(2, 4, 8)), dict(grad_gate=t(2, 5, 8, dtype=bf16)),
    dict(grad_h_last=t(2, 9)), dict(grad_h0=t(3, 8)), dict(lengths=t(1, dtype=torch.int32))])
def test_scan_bwd_binding_refuses(bad):
    a = dict(gate=t(2, 5, 8), x=t(2, 5, 8), states=t(16), grad_y=t(2, 5, 8), grad_gate=t(2, 5, 8), grad_x=t(2, 5, 8))
    a.update(bad)
    with pytest.raises(E):
        bc.gated_scan_bwd(**a)


@pytest.mark.parametrize("bad", [
    dict(x=t(2, 1, 8)), dict(gate=t(2, 7)), dict(gate=None), dict(y=t(3, 8)), dict(y=t(2, 8, dtype=bf16)),
    dict(state=t(4, 7)), dict(state=t(4, 8, dtype=bf16)), dict(state_out=t(3, 8)), dict(slots=t(2)),
    dict(slots=t(3, dtype=torch.int32))])
def test_scan_step_binding_refuses(bad):
    a = dict(gate=t(2, 8), x=t(2, 8), state=t(4, 8), y=t(2, 8))
    a.update(bad)
    with pytest.raises(E):
        bc.gated_scan_step(**a)


i8 = torch.int8


@pytest.mark.parametrize("bad", [
    dict(wq=t(3, 256, dtype=i8)), dict(wq=t(3, 128)), dict(wq=None), dict(w_scale=t(4)), dict(x=t(8)),
    dict(x=t(5, 8, dtype=f64)), dict(out=t(5, 4)), dict(out=t(5, 3, dtype=f64)), dict(out=None), dict(bias=t(4)),
    dict(layout=3), dict(x=t(5, 128, dtype=i8)), dict(x=t(5, 256, dtype=i8), x_scale=t(5)),
    dict(x=t(5, 128, dtype=i8), x_scale=t(4))])
def test_mix_i8_binding_refuses(bad):
    a = dict(wq=t(3, 128, dtype=i8), w_scale=t(3), x=t(5, 8), out=t(5, 3))
    a.update(bad)
    with pytest.raises(E):
        bc.pointwise_mix_i8(**a)


@pytest.mark.parametrize("bad", [dict(q=t(5, 256, dtype=i8)), dict(q=t(5, 128)), dict(scale=t(4)),
                                 dict(src=t(5, 8, dtype=f64)), dict(q=None)])
def test_quantize_binding_refuses(bad):
    a = dict(src=t(5, 8), q=t(5, 128, dtype=i8), scale=t(5))
    a.update(bad)
    with pytest.raises(E):
        bc.quantize_i8(**a)


# ---- the oracle itself -------------------------------------------------------

@pytest.mark.parametrize("form", ["logit", "value"])
@pytest.mark.parametrize("lengths", [None, [7, 0, 3]])
def test_oracle_gradients_are_the_losss_differences(form, lengths):
    """The loss is smooth in every argument: a central difference of step 1e-5
    in 64 bits is right to about 1e-9."""
    rng = np.random.default_rng(1)
    T, N, C = 7, 3, 4
    gate, x, gy = rng.standard_normal((3, T, N, C))
    h0, gh = rng.standard_normal((2, N, C))

    def loss(gate, x, h0):
        h, y, _ = R.scan_forward(gate, x, h0, lengths, form)
        return (y * gy).sum() + (h[T] * gh).sum()

    g = R.scan_backward(gate, x, gy, h0, gh, lengths, form)
    for name, i in (("gate", 0), ("x", 1), ("h0", 2)):
        v, eps = rng.standard_normal((gate, x, h0)[i].shape), 1e-5
        at = lambda s: loss(*[a + s * eps * v if k == i else a for k, a in enumerate((gate, x, h0))])
        assert abs((at(1) - at(-1)) / (2 * eps) - (g[name] * v).sum()) < 1e-7


def test_oracle_codes():
    q, s = R.codes(np.array([[2, 1, -2, 0.5], [0, 0, 0, 0], [np.nan, 1, 1, 1]], np.float32))
    assert q[0].tolist() == [127, 64, -127, 32] and q[1].tolist() == [0] * 4
    assert s[0] == np.float32(2) / np.float32(127) and s[1] == 0 and np.isnan(s[2])
