"""The binding of the recurrent layer's calls refuses a tensor of the wrong size,
type or strides by its name, before it asks where the tensors live: on CPU
tensors a call without a fault says that they are not on the GPU, and only that
call.  No GPU."""
import os

import pytest
import torch

from paper_1906_11367_amd import boxconv as bc

pytestmark = pytest.mark.skipif(not os.path.exists(bc.LIB_PATH), reason="libboxconv.so not built")

bf16, f64, i8, i32 = torch.bfloat16, torch.float64, torch.int8, torch.int32


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


STATES = 16   # 2 sequences of 8 channels, one kept state
CALLS = {
    "gated_scan_fwd": dict(gate=t(2, 5, 8), x=t(2, 5, 8), y=t(2, 5, 8), h0=t(2, 8), h_last=t(2, 8),
                           lengths=t(2, dtype=i32), states=t(STATES)),
    "gated_scan_bwd": dict(gate=t(2, 5, 8), x=t(2, 5, 8), states=t(STATES), grad_y=t(2, 5, 8), grad_gate=t(2, 5, 8),
                           grad_x=t(2, 5, 8), grad_h_last=t(2, 8), grad_h0=t(2, 8), lengths=t(2, dtype=i32)),
    "gated_scan_step": dict(gate=t(2, 8), x=t(2, 8), state=t(4, 8), y=t(2, 8), slots=t(2, dtype=i32),
                            state_out=t(4, 8)),
    "quantize_i8": dict(src=t(5, 8), q=t(5, 128, dtype=i8), scale=t(5)),
    "pointwise_mix_i8": dict(wq=t(3, 128, dtype=i8), w_scale=t(3), x=t(5, 8), out=t(5, 3), bias=t(3)),
}


@pytest.mark.parametrize("call", CALLS)
def test_a_call_without_a_fault_asks_for_the_gpu(call):
    with pytest.raises(bc.BoxConvError, match="must be on the GPU"):
        getattr(bc, call)(**CALLS[call])


@pytest.mark.parametrize("call,bad,says", [
    ("gated_scan_fwd", dict(gate=t(2, 5, 7)), "gate has shape"),
    ("gated_scan_fwd", dict(gate=t(2, 5, 8, dtype=bf16)), "gate has dtype"),
    ("gated_scan_fwd", dict(gate=t(2, 5, 9)[..., :8]), "same strides"),
    ("gated_scan_fwd", dict(gate=t(2, 8, 5).transpose(1, 2), x=t(2, 8, 5).transpose(1, 2)), "gate must be contiguous"),
    ("gated_scan_fwd", dict(x=t(2, 40)), "x must be a 3-D"), ("gated_scan_fwd", dict(x=t(2, 5, 8, dtype=f64)), "x has dtype"),
    ("gated_scan_fwd", dict(y=t(2, 5, 9)), "y has shape"), ("gated_scan_fwd", dict(y=t(2, 5, 8, dtype=f64)), "y has dtype"),
    ("gated_scan_fwd", dict(h0=t(2, 7)), "h0 has shape"), ("gated_scan_fwd", dict(h_last=t(2, 8, dtype=bf16)), "h_last has dtype"),
    ("gated_scan_fwd", dict(lengths=t(2)), "lengths has dtype"), ("gated_scan_fwd", dict(lengths=t(3, dtype=i32)), "lengths has shape"),
    ("gated_scan_fwd", dict(states=t(3)), "states has 3 elements"), ("gated_scan_fwd", dict(layout=4), "unknown layout"),
    ("gated_scan_bwd", dict(grad_y=t(2, 5, 9)), "grad_y has shape"), ("gated_scan_bwd", dict(grad_y=t(2, 5, 8, dtype=bf16)), "grad_y has dtype"),
    ("gated_scan_bwd", dict(grad_x=t(2, 4, 8)), "grad_x has shape"), ("gated_scan_bwd", dict(grad_gate=t(2, 5, 8, dtype=bf16)), "grad_gate has dtype"),
    ("gated_scan_bwd", dict(grad_gate=t(2, 5, 9)[..., :8]), "same strides"), ("gated_scan_bwd", dict(grad_h_last=t(2, 9)), "grad_h_last has shape"),
    ("gated_scan_bwd", dict(grad_h0=t(3, 8)), "grad_h0 has shape"), ("gated_scan_bwd", dict(states=t(15)), "states has 15 elements"),
    ("gated_scan_step", dict(gate=t(2, 7)), "gate has shape"), ("gated_scan_step", dict(gate=t(2, 9)[:, :8]), "same strides"),
    ("gated_scan_step", dict(y=t(3, 8)), "y has shape"), ("gated_scan_step", dict(state=t(4, 7)), "state has shape"),
    ("gated_scan_step", dict(state=t(4, 8, dtype=bf16)), "state has dtype"), ("gated_scan_step", dict(state_out=t(3, 8)), "state_out has shape"),
    ("gated_scan_step", dict(slots=t(2)), "slots has dtype"), ("gated_scan_step", dict(slots=t(3, dtype=i32)), "slots has shape"),
    ("quantize_i8", dict(q=t(5, 256, dtype=i8)), "q has shape"), ("quantize_i8", dict(q=t(5, 128)), "q has dtype"),
    ("quantize_i8", dict(q=t(4, 128, dtype=i8)), "q has shape"), ("quantize_i8", dict(scale=t(4)), "scale has shape"),
    ("quantize_i8", dict(src=t(5, 8, dtype=f64)), "src must be"), ("quantize_i8", dict(src=t(5, 16)[:, ::2]), "src must be contiguous"),
    ("pointwise_mix_i8", dict(wq=t(3, 256, dtype=i8)), "wq has rows of 256"), ("pointwise_mix_i8", dict(wq=t(3, 128)), "wq must be"),
    ("pointwise_mix_i8", dict(w_scale=t(4)), "w_scale has shape"), ("pointwise_mix_i8", dict(out=t(5, 4)), "out has shape"),
    ("pointwise_mix_i8", dict(out=t(4, 3)), "out has shape"), ("pointwise_mix_i8", dict(out=t(5, 3, dtype=f64)), "out must be"),
    ("pointwise_mix_i8", dict(bias=t(4)), "bias has shape"), ("pointwise_mix_i8", dict(layout=3), "unknown layout"),
    ("pointwise_mix_i8", dict(x=t(8)), "x must be"), ("pointwise_mix_i8", dict(x=t(5, 128, dtype=i8)), "codes need x_scale"),
    ("pointwise_mix_i8", dict(x=t(5, 256, dtype=i8), x_scale=t(5)), "x has shape"),
    ("pointwise_mix_i8", dict(x=t(5, 128, dtype=i8), x_scale=t(4)), "x_scale has shape"),
    ("pointwise_mix_i8", dict(x=t(5, 8, 1)[..., 0].t(), out=t(8, 3)), "x must be contiguous"),
    ("pointwise_mix_i8", dict(x=t(2, 8, 6), layout=bc.BC_MAPS, out=t(2, 3, 5)), "out has shape"),
    ("pointwise_mix_i8", dict(x=t(5, 128, dtype=i8), x_scale=t(5), layout=bc.BC_MAPS, out=t(2, 3, 2)), "are not 2 maps")])
def test_refusals_name_their_argument(call, bad, says):
    with pytest.raises(bc.BoxConvError, match=f"^{call}: .*{says}"):
        getattr(bc, call)(**{**CALLS[call], **bad})


@pytest.mark.parametrize("call,missing", [
    ("gated_scan_fwd", "gate x y"), ("gated_scan_bwd", "gate x states grad_y grad_gate grad_x"),
    ("gated_scan_step", "gate x state y"), ("quantize_i8", "src q scale"), ("pointwise_mix_i8", "wq w_scale x out")])
def test_what_a_call_needs_is_asked_for(call, missing):
    for name in missing.split():
        with pytest.raises(bc.BoxConvError, match=f"^{call}: .*{name}"):
            getattr(bc, call)(**{**CALLS[call], name: None})


def test_an_output_without_dimensions():
    with pytest.raises(bc.BoxConvError, match="out has shape"):
        bc.pointwise_mix_i8(**{**CALLS["pointwise_mix_i8"], "x": t(1, 8), "wq": t(1, 128, dtype=i8), "w_scale": t(1),
                               "bias": None, "out": t()})


def test_an_output_without_dimensions_for_codes_of_maps():
    with pytest.raises(bc.BoxConvError, match="5 rows of codes are not 0 maps"):
        bc.pointwise_mix_i8(**{**CALLS["pointwise_mix_i8"], "x": t(5, 128, dtype=i8), "x_scale": t(5),
                               "layout": bc.BC_MAPS, "out": t()})


def test_maps_of_one_column():
    """Contiguous maps [N, K, H, 1] whose last stride says nothing."""
    x = t(2, 8, 1, 5).transpose(2, 3)
    assert x.stride() == (40, 5, 1, 5) and x.is_contiguous()
    call = {**CALLS["pointwise_mix_i8"], "x": x, "layout": bc.BC_MAPS, "out": t(2, 3, 5)}
    with pytest.raises(bc.BoxConvError, match="must be on the GPU"):
        bc.pointwise_mix_i8(**call)
    with pytest.raises(bc.BoxConvError, match="x's maps must be contiguous"):
        bc.pointwise_mix_i8(**{**call, "x": t(2, 8, 5, 4)[..., :1]})


@pytest.mark.gpu
def test_maps_of_one_column_are_read_as_they_stand():
    g = torch.Generator().manual_seed(1)
    x = torch.randn((2, 8, 1, 5), generator=g).cuda().transpose(2, 3)
    wq, ws = bc.quantize_i8(torch.randn((3, 8), generator=g).cuda(), torch.empty((3, 128), dtype=i8, device="cuda"),
                            torch.empty(3, device="cuda"))
    out, want = torch.empty((2, 3, 5), device="cuda"), torch.empty((2, 3, 5), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, out, layout=bc.BC_MAPS)
    bc.pointwise_mix_i8(wq, ws, x.reshape(2, 8, 5).clone(), want, layout=bc.BC_MAPS)
    assert torch.equal(out, want) and torch.isfinite(out).all()


@pytest.mark.parametrize("gone", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_the_stream_without_torchs_own_functions(monkeypatch, gone):
    """Every entry point asks for the current stream; it is the public one where a
    torch does not have the shorter way."""
    class Stream:
        cuda_stream = 0x5000

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x7000, raising=False)
    assert bc._stream() == 0x7000
    monkeypatch.delattr(torch._C, gone)
    assert bc._stream() == 0x5000


@pytest.mark.gpu
def test_the_stream_is_torchs_current_one():
    side = torch.cuda.Stream()
    assert bc._stream() == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert bc._stream() == side.cuda_stream
