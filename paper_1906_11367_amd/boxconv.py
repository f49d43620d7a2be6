"""Thin ctypes binding of libboxconv.so (C ABI: include/boxconv.h).

Argument marshalling only: tensors are passed as device pointers together with
torch's current HIP stream; every step of the layer runs in the library's
kernels.  The library is required: if it is not built, or a GPU is not
present, the calls raise -- there is no fallback implementation.

Entry points (same names as the C ABI): box_prep, sat_build, box_conv_fwd,
box_conv_bwd, box_conv_fwd_strided, box_conv_bwd_strided, pointwise_mix, the
box-parameter reparameterisation (box_params_from_unit, box_params_unit_grad,
box_params_clip), kernel splitting (box_conv_split_fwd, box_conv_split_bwd),
the bf16 helpers (bc_cast_bf16, bc_relu_grad_bf16), the gated scan of
recurrent layers (gated_scan_fwd, gated_scan_bwd, gated_scan_step), the 8-bit
mix (quantize_i8, pointwise_mix_i8), linear attention (linear_attention_fwd,
linear_attention_bwd, linear_attention_step), the norms around a block
(block_norm_fwd, block_norm_bwd), plus the workspace-size queries.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libboxconv.so")

BC_I32, BC_F32, BC_BF16, BC_I8 = 0, 1, 2, 3
BC_MIX_FWD, BC_MIX_BWD_DATA, BC_MIX_BWD_WEIGHT = 0, 1, 2
BC_FLAG_MEAN_OFFSET, BC_FLAG_FORCE_HBM, BC_FLAG_INTEGER_CORNERS = 1, 2, 4
BC_SPLIT_2X, BC_SPLIT_2Y, BC_SPLIT_4 = 1, 2, 3
BC_SPLIT_FORCE_HBM = 0x100
BC_TOKENS, BC_MAPS = 0, 1
BC_GATE_LOGIT, BC_GATE_VALUE, BC_GATE_LOG = 0, 1, 2
BC_NORM_RMS, BC_NORM_LAYER = 0, 1
BC_ACT_SILU, BC_ACT_SIGMOID = 0, 1
STATUS = {0: "BC_OK", 1: "BC_ERR_NULL", 2: "BC_ERR_SHAPE", 3: "BC_ERR_DTYPE", 4: "BC_ERR_ALIGN",
          5: "BC_ERR_WORKSPACE", 6: "BC_ERR_HIP", 7: "BC_ERR_UNSUPPORTED"}

# Exported symbols and their C signatures (kept in step with boxconv.h).
_vp, _i, _u, _sz, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint, ctypes.c_size_t, ctypes.c_float
_ll = ctypes.c_int64


class bc_strides(ctypes.Structure):
    _fields_ = [("batch", _ll), ("row", _ll), ("head", _ll)]


class bc_attention(ctypes.Structure):
    _fields_ = [(n, _i) for n in ("N", "T", "H", "Hq", "Hk", "Hv", "Dk", "Dv", "dt", "gate_dt", "form")] + [("scale", _f)]


class bc_norm(ctypes.Structure):
    _fields_ = [(n, _i) for n in ("R", "C", "groups", "kind", "act", "dt")] + [("eps", _f)]


_st, _at, _nm = bc_strides, ctypes.POINTER(bc_attention), ctypes.POINTER(bc_norm)
SIGNATURES = {
    "box_prep": (_i, [_vp, _i, _i, _u, _vp, _vp]),
    "sat_build": (_i, [_vp, _i, _vp, _vp, _i, _i, _i, _i, _vp]),
    "box_conv_fwd": (_i, [_vp, _i, _vp, _i, _i, _i, _i, _i, _vp, _i, _u, _vp, _sz, _vp]),
    "box_conv_bwd": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _u, _vp, _sz, _vp]),
    "box_conv_fwd_strided": (_i, [_vp, _i, _vp, _i, _i, _i, _i, _i, _i, _vp, _i, _u, _vp, _sz, _vp]),
    "box_params_from_unit": (_i, [_vp, _i, _i, _f, _f, _vp, _vp]),
    "box_params_unit_grad": (_i, [_vp, _i, _i, _f, _f, _vp, _vp]),
    "box_params_clip": (_i, [_vp, _i, _i, _vp]),
    "box_conv_bwd_strided": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _u, _vp, _sz, _vp]),
    "pointwise_mix": (_i, [_i, _vp, _i, _vp, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _vp, _sz, _vp]),
    "box_conv_split_fwd": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _i, _vp, _sz, _vp]),
    "box_conv_split_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bc_split_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "bc_box_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _u]),
    "bc_box_workspace_bytes_strided": (_sz, [_i, _i, _i, _i, _i, _i, _i, _u]),
    "bc_mix_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "bc_cast_bf16": (_i, [_vp, _vp, _sz, _vp]),
    "bc_relu_grad_bf16": (_i, [_vp, _vp, _vp, _sz, _vp]),
    "box_conv_bwd_relu_bf16": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _u, _vp, _sz, _vp]),
    "box_conv_bwd_noalloc": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _u, _vp]),
    "bc_noalloc_scratch_bytes": (_sz, []),
    "gated_scan_fwd": (_i, [_vp, _vp, _i, _ll, _ll, _vp, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _i, _vp, _sz, _vp]),
    "gated_scan_bwd": (_i, [_vp, _vp, _i, _ll, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _i, _ll, _ll, _vp, _i, _i, _i, _i,
                            _i, _vp, _sz, _vp]),
    "gated_scan_step": (_i, [_vp, _vp, _i, _ll, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "bc_gated_scan_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "bc_gated_scan_states_bytes": (_sz, [_i, _i, _i, _i]),
    "quantize_i8": (_i, [_vp, _i, _ll, _ll, _vp, _vp, _i, _i, _i, _i, _vp]),
    "pointwise_mix_i8": (_i, [_vp, _vp, _vp, _i, _ll, _ll, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _sz, _vp]),
    "bc_i8_pitch": (_i, [_i]),
    "bc_mix_i8_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "linear_attention_fwd": (_i, [_at, _vp, _st, _vp, _st, _vp, _st, _vp, _st, _vp, _vp, _vp, _st, _vp, _vp, _vp, _sz, _vp]),
    "linear_attention_bwd": (_i, [_at, _vp, _st, _vp, _st, _vp, _st, _vp, _st, _vp, _vp, _vp, _st, _vp, _vp, _st, _vp, _st,
                                  _vp, _st, _vp, _st, _vp, _vp, _sz, _vp]),
    "linear_attention_step": (_i, [_at, _vp, _st, _vp, _st, _vp, _st, _vp, _st, _vp, _vp, _vp, _vp, _i, _vp]),
    "bc_linear_attention_workspace_bytes": (_sz, [_i, _at]),
    "bc_linear_attention_states_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "block_norm_fwd": (_i, [_nm, _vp, _ll, _vp, _ll, _vp, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp]),
    "block_norm_bwd": (_i, [_nm, _vp, _ll, _vp, _ll, _vp, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _ll, _vp, _ll, _vp,
                            _ll, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bc_block_norm_workspace_bytes": (_sz, [_i, _i]),
    "bc_status_string": (ctypes.c_char_p, [_i]),
    "bc_abi_version": (_i, []),
}

_lib = None


class BoxConvError(RuntimeError):
    pass


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads libboxconv.so (no GPU needed to load it)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise BoxConvError(f"{path} is not built: run `python -m paper_1906_11367_amd.build` "
                           "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        msg = load_library().bc_status_string(status).decode()
        raise BoxConvError(f"{what}: {STATUS.get(status, status)} ({msg})")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise BoxConvError("tensors must be on the GPU")
    if not t.is_contiguous():
        raise BoxConvError("tensors must be contiguous")
    return t.data_ptr()


def _need(t, shape, dtypes, what, name):
    """Shape and dtype checks the C ABI cannot make (it sees only pointers):
    a tensor of the wrong size or type would be read or written out of bounds
    on the device.  shape entries of None match any extent."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise BoxConvError(f"{what}: {name} must be a tensor")
    # the common case first: a small call is bound by this marshalling
    if (t.dtype is dtypes or (type(dtypes) is tuple and t.dtype in dtypes)) and (shape is None or t.shape == shape):
        return
    if isinstance(dtypes, torch.dtype):
        dtypes = (dtypes,)
    if t.dtype not in dtypes:
        raise BoxConvError(f"{what}: {name} has dtype {t.dtype}, expected one of {tuple(dtypes)}")
    if shape is not None:
        if t.dim() != len(shape) or any(e is not None and int(a) != int(e) for a, e in zip(t.shape, shape)):
            raise BoxConvError(f"{what}: {name} has shape {tuple(t.shape)}, expected "
                               f"{tuple('*' if e is None else e for e in shape)}")


def _need_numel(t, n, dtypes, what, name):
    if isinstance(dtypes, torch.dtype):
        dtypes = (dtypes,)
    if t.dtype not in dtypes:
        raise BoxConvError(f"{what}: {name} has dtype {t.dtype}, expected one of {tuple(dtypes)}")
    if t.numel() != n:
        raise BoxConvError(f"{what}: {name} has {t.numel()} elements, expected {n}")


_MAPS = (torch.int32, torch.float32)
_F32 = torch.float32


def _maps_and_boxes(x, boxes, what):
    if not isinstance(x, torch.Tensor) or x.dim() != 4:
        raise BoxConvError(f"{what}: x must be a 4-D [N, C, H, W] tensor")
    _need(x, None, _MAPS, what, "x")
    N, C, H, W = x.shape
    B = boxes.shape[1] if isinstance(boxes, torch.Tensor) and boxes.dim() == 3 else None
    _need(boxes, (C, B, 4), _F32, what, "boxes")
    return N, C, H, W, B


def _stream():
    # the current device's current stream, without building a Stream object (a
    # microsecond of a small call) where torch has the functions its own
    # Stream is made from; they are not part of its interface
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.int32:
        return BC_I32
    if t.dtype == torch.float32:
        return BC_F32
    if t.dtype == torch.bfloat16:
        return BC_BF16
    if t.dtype == torch.int8:
        return BC_I8
    raise BoxConvError(f"unsupported dtype {t.dtype}")


def _workspace(nbytes: int, device) -> torch.Tensor | None:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def box_workspace_bytes(op: int, N, C, H, W, B, flags=0, stride: int = 1) -> int:
    return int(load_library().bc_box_workspace_bytes_strided(op, N, C, H, W, B, stride, flags))


def mix_workspace_bytes(mode: int, N, M, K, P, compute_dt) -> int:
    return int(load_library().bc_mix_workspace_bytes(mode, N, M, K, P, compute_dt))


def box_prep(boxes: torch.Tensor, table: torch.Tensor, flags: int = 0):
    """table: int32 tensor of 2*C*B*16 words (see boxconv.h)."""
    _need(boxes, (None, None, 4), _F32, "box_prep", "boxes")
    C, B = boxes.shape[0], boxes.shape[1]
    _need_numel(table, 2 * C * B * 16, torch.int32, "box_prep", "table")
    _check(load_library().box_prep(_ptr(boxes), C, B, flags, _ptr(table), _stream()), "box_prep")
    return table


def sat_build(x: torch.Tensor, sat: torch.Tensor, mean: torch.Tensor | None = None):
    """x [N, C, H, W] int32/fp32 -> sat [N, C, H+1, W+1] (exclusive table)."""
    if not isinstance(x, torch.Tensor) or x.dim() != 4:
        raise BoxConvError("sat_build: x must be a 4-D [N, C, H, W] tensor")
    _need(x, None, _MAPS, "sat_build", "x")
    N, C, H, W = x.shape
    _need(sat, (N, C, H + 1, W + 1), x.dtype, "sat_build", "sat")
    _need(mean, (N, C), _F32, "sat_build", "mean")
    _check(load_library().sat_build(_ptr(x), dtype_code(x), _ptr(sat), _ptr(mean), N, C, H, W, _stream()),
           "sat_build")
    return sat


def _strided_shape(N, C, H, W, B, stride):
    return (N, C * B, (H + stride - 1) // stride, (W + stride - 1) // stride)


def box_conv_fwd(x: torch.Tensor, boxes: torch.Tensor, y: torch.Tensor, flags: int = 0,
                 ws: torch.Tensor | None = None, stride: int = 1):
    """x [N, C, H, W], boxes [C, B, 4] fp32 -> y [N, C*B, ceil(H/stride), ceil(W/stride)]
    (int32, fp32 or bf16); stride > 1 calls box_conv_fwd_strided."""
    N, C, H, W, B = _maps_and_boxes(x, boxes, "box_conv_fwd")
    _need(y, _strided_shape(N, C, H, W, B, stride),
          torch.int32 if x.dtype == torch.int32 else (torch.float32, torch.bfloat16), "box_conv_fwd", "y")
    if ws is None:
        ws = _workspace(box_workspace_bytes(0, N, C, H, W, B, flags, stride), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    lib = load_library()
    if stride == 1:
        st = lib.box_conv_fwd(_ptr(x), dtype_code(x), _ptr(boxes), N, C, H, W, B, _ptr(y), dtype_code(y), flags,
                              _ptr(ws), nbytes, _stream())
    else:
        st = lib.box_conv_fwd_strided(_ptr(x), dtype_code(x), _ptr(boxes), N, C, H, W, B, stride, _ptr(y),
                                      dtype_code(y), flags, _ptr(ws), nbytes, _stream())
    _check(st, "box_conv_fwd")
    return y


def box_conv_fwd_strided(x, boxes, stride: int, y, flags: int = 0, ws=None):
    return box_conv_fwd(x, boxes, y, flags, ws, stride)


def box_conv_bwd(x: torch.Tensor, boxes: torch.Tensor, grad_y: torch.Tensor, grad_x: torch.Tensor | None,
                 grad_boxes: torch.Tensor | None, flags: int = 0, ws: torch.Tensor | None = None, stride: int = 1):
    """grad_y [N, C*B, ceil(H/stride), ceil(W/stride)]; stride > 1 calls box_conv_bwd_strided."""
    N, C, H, W, B = _maps_and_boxes(x, boxes, "box_conv_bwd")
    _need(x, None, _F32, "box_conv_bwd", "x")
    _need(grad_y, _strided_shape(N, C, H, W, B, stride), _F32, "box_conv_bwd", "grad_y")
    _need(grad_x, (N, C, H, W), _F32, "box_conv_bwd", "grad_x")
    _need(grad_boxes, (C, B, 4), _F32, "box_conv_bwd", "grad_boxes")
    if ws is None:
        ws = _workspace(box_workspace_bytes(1, N, C, H, W, B, flags, stride), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    lib = load_library()
    if stride == 1:
        st = lib.box_conv_bwd(_ptr(x), _ptr(boxes), _ptr(grad_y), N, C, H, W, B, _ptr(grad_x), _ptr(grad_boxes),
                              flags, _ptr(ws), nbytes, _stream())
    else:
        st = lib.box_conv_bwd_strided(_ptr(x), _ptr(boxes), _ptr(grad_y), N, C, H, W, B, stride, _ptr(grad_x),
                                      _ptr(grad_boxes), flags, _ptr(ws), nbytes, _stream())
    _check(st, "box_conv_bwd")
    return grad_x, grad_boxes


def box_conv_bwd_relu_bf16(x: torch.Tensor, boxes: torch.Tensor, grad_y: torch.Tensor,
                           grad_x_bf16: torch.Tensor | None, grad_boxes: torch.Tensor | None, flags: int = 0,
                           ws: torch.Tensor | None = None, stride: int = 1):
    """As box_conv_bwd, with the input gradient written as bf16(x > 0 ? dL/dx : 0)
    (x: the rectified output of a bf16 mix before this layer)."""
    what = "box_conv_bwd_relu_bf16"
    N, C, H, W, B = _maps_and_boxes(x, boxes, what)
    _need(x, None, _F32, what, "x")
    _need(grad_y, _strided_shape(N, C, H, W, B, stride), _F32, what, "grad_y")
    _need(grad_x_bf16, (N, C, H, W), torch.bfloat16, what, "grad_x")
    _need(grad_boxes, (C, B, 4), _F32, what, "grad_boxes")
    if ws is None:
        ws = _workspace(box_workspace_bytes(1, N, C, H, W, B, flags, stride), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(load_library().box_conv_bwd_relu_bf16(_ptr(x), _ptr(boxes), _ptr(grad_y), N, C, H, W, B, stride,
                                                 _ptr(grad_x_bf16), _ptr(grad_boxes), flags, _ptr(ws), nbytes,
                                                 _stream()), "box_conv_bwd_relu_bf16")
    return grad_x_bf16, grad_boxes


def box_conv_bwd_noalloc(x: torch.Tensor, boxes: torch.Tensor, grad_y: torch.Tensor, grad_x: torch.Tensor | None,
                         grad_boxes: torch.Tensor | None, flags: int = 0):
    """box_conv_bwd with the library's own fixed scratch array as workspace:
    the call allocates nothing (bc_noalloc_scratch_bytes() is the limit)."""
    what = "box_conv_bwd_noalloc"
    N, C, H, W, B = _maps_and_boxes(x, boxes, what)
    _need(x, None, _F32, what, "x")
    _need(grad_y, (N, C * B, H, W), _F32, what, "grad_y")
    _need(grad_x, (N, C, H, W), _F32, what, "grad_x")
    _need(grad_boxes, (C, B, 4), _F32, what, "grad_boxes")
    _check(load_library().box_conv_bwd_noalloc(_ptr(x), _ptr(boxes), _ptr(grad_y), N, C, H, W, B, _ptr(grad_x),
                                               _ptr(grad_boxes), flags, _stream()), what)
    return grad_x, grad_boxes


def noalloc_scratch_bytes() -> int:
    return int(load_library().bc_noalloc_scratch_bytes())


def box_conv_bwd_strided(x, boxes, grad_y, stride: int, grad_x, grad_boxes, flags: int = 0, ws=None):
    return box_conv_bwd(x, boxes, grad_y, grad_x, grad_boxes, flags, ws, stride)


def box_params_from_unit(u: torch.Tensor, max_w: float, max_h: float, boxes: torch.Tensor):
    """u [C, B, 4] unit corners -> boxes [C, B, 4] (cx, cy, rx, ry) in pixels."""
    _need(u, (None, None, 4), _F32, "box_params_from_unit", "u")
    C, B = u.shape[0], u.shape[1]
    _need(boxes, (C, B, 4), _F32, "box_params_from_unit", "boxes")
    _check(load_library().box_params_from_unit(_ptr(u), C, B, max_w, max_h, _ptr(boxes), _stream()),
           "box_params_from_unit")
    return boxes


def box_params_unit_grad(grad_boxes: torch.Tensor, max_w: float, max_h: float, grad_u: torch.Tensor):
    _need(grad_boxes, (None, None, 4), _F32, "box_params_unit_grad", "grad_boxes")
    C, B = grad_boxes.shape[0], grad_boxes.shape[1]
    _need(grad_u, (C, B, 4), _F32, "box_params_unit_grad", "grad_u")
    _check(load_library().box_params_unit_grad(_ptr(grad_boxes), C, B, max_w, max_h, _ptr(grad_u), _stream()),
           "box_params_unit_grad")
    return grad_u


def box_params_clip(u: torch.Tensor):
    _need(u, (None, None, 4), _F32, "box_params_clip", "u")
    C, B = u.shape[0], u.shape[1]
    _check(load_library().box_params_clip(_ptr(u), C, B, _stream()), "box_params_clip")
    return u


SPLIT_MODES = {"2x": BC_SPLIT_2X, "2y": BC_SPLIT_2Y, "4": BC_SPLIT_4}
SPLIT_PIECES = {BC_SPLIT_2X: 2, BC_SPLIT_2Y: 2, BC_SPLIT_4: 4}


def _split_mode(mode) -> int:
    m = SPLIT_MODES.get(mode, mode)
    if m not in SPLIT_PIECES:
        raise BoxConvError(f"unknown split mode {mode!r}")
    return m


def split_workspace_bytes(op: int, N, C, H, W, B, mode, force_hbm: bool = False) -> int:
    code = _split_mode(mode) | (BC_SPLIT_FORCE_HBM if force_hbm else 0)
    return int(load_library().bc_split_workspace_bytes(op, N, C, H, W, B, code))


def box_conv_split_fwd(x: torch.Tensor, boxes: torch.Tensor, piece_w: torch.Tensor, mode, y: torch.Tensor,
                       ws: torch.Tensor | None = None, force_hbm: bool = False):
    """x [N, C, H, W] fp32, boxes [C, B, 4], piece_w [C, B, P] -> y [N, C*B, H, W] (fp32 or bf16).
    mode: "2x", "2y", "4" or a BC_SPLIT_* code; force_hbm: take the HBM-table
    kernels even where the map's table fits in LDS."""
    m = _split_mode(mode)
    code = m | (BC_SPLIT_FORCE_HBM if force_hbm else 0)
    what = "box_conv_split_fwd"
    N, C, H, W, B = _maps_and_boxes(x, boxes, what)
    _need(x, None, _F32, what, "x")
    _need(piece_w, (C, B, SPLIT_PIECES[m]), _F32, what, "piece_w")
    _need(y, (N, C * B, H, W), (torch.float32, torch.bfloat16), what, "y")
    if ws is None:
        ws = _workspace(split_workspace_bytes(0, N, C, H, W, B, m, force_hbm), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(load_library().box_conv_split_fwd(_ptr(x), _ptr(boxes), _ptr(piece_w), N, C, H, W, B, code, _ptr(y),
                                             dtype_code(y), _ptr(ws), nbytes, _stream()), "box_conv_split_fwd")
    return y


def box_conv_split_bwd(x: torch.Tensor, boxes: torch.Tensor, piece_w: torch.Tensor, mode, grad_y: torch.Tensor,
                       grad_x: torch.Tensor | None, grad_boxes: torch.Tensor | None,
                       grad_w: torch.Tensor | None, ws: torch.Tensor | None = None, force_hbm: bool = False):
    m = _split_mode(mode)
    code = m | (BC_SPLIT_FORCE_HBM if force_hbm else 0)
    what = "box_conv_split_bwd"
    N, C, H, W, B = _maps_and_boxes(x, boxes, what)
    _need(x, None, _F32, what, "x")
    _need(piece_w, (C, B, SPLIT_PIECES[m]), _F32, what, "piece_w")
    _need(grad_y, (N, C * B, H, W), _F32, what, "grad_y")
    _need(grad_x, (N, C, H, W), _F32, what, "grad_x")
    _need(grad_boxes, (C, B, 4), _F32, what, "grad_boxes")
    _need(grad_w, (C, B, SPLIT_PIECES[m]), _F32, what, "grad_w")
    if ws is None:
        ws = _workspace(split_workspace_bytes(1, N, C, H, W, B, m, force_hbm), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(load_library().box_conv_split_bwd(_ptr(x), _ptr(boxes), _ptr(piece_w), _ptr(grad_y), N, C, H, W, B, code,
                                             _ptr(grad_x), _ptr(grad_boxes), _ptr(grad_w), _ptr(ws), nbytes,
                                             _stream()), "box_conv_split_bwd")
    return grad_x, grad_boxes, grad_w


def bc_cast_bf16(src: torch.Tensor, dst: torch.Tensor):
    """dst (bf16, same numel) = src (fp32) rounded to nearest even."""
    _need_numel(src, src.numel(), _F32, "bc_cast_bf16", "src")
    _need_numel(dst, src.numel(), torch.bfloat16, "bc_cast_bf16", "dst")
    _check(load_library().bc_cast_bf16(_ptr(src), _ptr(dst), src.numel(), _stream()), "bc_cast_bf16")
    return dst


def need_weights(w: torch.Tensor, n: int):
    """The checks bc_cast_bf16 makes of n fp32 weights, where no cast is made."""
    _need_numel(w, n, _F32, "pointwise_mix", "w")


def relu_grad_bf16(grad: torch.Tensor, out: torch.Tensor, dst: torch.Tensor):
    """dst (bf16) = bf16(out > 0 ? grad : 0): the ReLU backward in the mix's compute type."""
    if not (grad.numel() == out.numel() == dst.numel()):
        raise BoxConvError("bc_relu_grad_bf16: size mismatch")
    if grad.dtype != torch.float32 or out.dtype != torch.float32 or dst.dtype != torch.bfloat16:
        raise BoxConvError("bc_relu_grad_bf16: grad and out fp32, dst bf16")
    _check(load_library().bc_relu_grad_bf16(_ptr(grad), _ptr(out), _ptr(dst), grad.numel(), _stream()),
           "bc_relu_grad_bf16")
    return dst


def pointwise_mix(mode: int, a: torch.Tensor, b: torch.Tensor, out: torch.Tensor, N: int, M: int, K: int,
                  P: int, compute_dt: int, relu: int = 0, aux: torch.Tensor | None = None,
                  accumulate: int = 0, ws: torch.Tensor | None = None):
    """The 1x1 mix (include/boxconv.h): FWD out[N,M,P] = a[M,K] * b[N,K,P];
    BWD_DATA out[N,K,P] = a[M,K]^T * b[N,M,P]; BWD_WEIGHT out[M,K] (+)=
    sum_n a[N,M,P] * b[N,K,P]^T.  aux: the FWD output Z [N,M,P] (ReLU mask)."""
    what = "pointwise_mix"
    sizes = {BC_MIX_FWD: (M * K, N * K * P, N * M * P), BC_MIX_BWD_DATA: (M * K, N * M * P, N * K * P),
             BC_MIX_BWD_WEIGHT: (N * M * P, N * K * P, M * K)}
    if mode not in sizes:
        raise BoxConvError(f"{what}: unknown mode {mode}")
    na, nb, no = sizes[mode]
    operand = (torch.int32, torch.float32, torch.bfloat16)
    _need_numel(a, na, operand, what, "a")
    _need_numel(b, nb, operand, what, "b")
    _need_numel(out, no, (torch.int32, torch.float32), what, "out")
    if aux is not None:
        _need_numel(aux, N * M * P, _F32, what, "aux")
    if ws is None:
        ws = _workspace(mix_workspace_bytes(mode, N, M, K, P, compute_dt), a.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(load_library().pointwise_mix(mode, _ptr(a), dtype_code(a), _ptr(b), dtype_code(b), _ptr(out),
                                        dtype_code(out), N, M, K, P, compute_dt, relu, _ptr(aux), accumulate,
                                        _ptr(ws), nbytes, _stream()), "pointwise_mix")
    return out


# ---- recurrent layers ---------------------------------------------------------

_FLOATS = (torch.float32, torch.bfloat16)


def _data(t: torch.Tensor):
    """The pointer of a tensor whose strides are passed along."""
    if not t.is_cuda:
        raise BoxConvError("tensors must be on the GPU")
    return t.data_ptr()


def _rows(t: torch.Tensor, what: str, name: str):
    """Batch stride and row stride of a 3-D tensor whose last dimension is
    contiguous (a slice of a larger tensor, for one).  Strides of dimensions of
    one element are the contiguous ones."""
    if not isinstance(t, torch.Tensor):
        raise BoxConvError(f"{what}: {name} must be a tensor")
    n, r, c = t.shape
    sn, sr, sc = t.stride()
    if sc != 1 and c > 1:
        raise BoxConvError(f"{what}: {name} must be contiguous in its last dimension")
    if r == 1:
        sr = c
    return (sn if n > 1 else sr * r), sr


_CODES = {torch.int32: BC_I32, torch.float32: BC_F32, torch.bfloat16: BC_BF16, torch.int8: BC_I8}


def _seq_sizes(x, layout, what):
    """N, T, C of a sequence tensor in its layout."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise BoxConvError(f"{what}: x must be a 3-D tensor")
    if x.dtype not in _FLOATS:
        raise BoxConvError(f"{what}: x has dtype {x.dtype}, expected one of {_FLOATS}")
    if layout == BC_TOKENS:
        return x.shape
    if layout == BC_MAPS:
        return x.shape[0], x.shape[2], x.shape[1]
    raise BoxConvError(f"{what}: unknown layout {layout}")


def _out_types(dtype):
    return _FLOATS if dtype is torch.float32 else (dtype,)


def gated_scan_workspace_bytes(op: int, N, T, C, dt: int, layout: int = BC_TOKENS) -> int:
    """op: 0 = gated_scan_fwd, 1 = gated_scan_bwd; dt: dtype code of gate and x."""
    return int(load_library().bc_gated_scan_workspace_bytes(op, N, T, C, dt, layout))


def gated_scan_states(N, T, C, dtype=None, layout: int = BC_TOKENS, device="cuda") -> torch.Tensor:
    """The buffer in which gated_scan_fwd keeps what gated_scan_bwd starts from
    (its layout is the library's; fp32 whatever the tensors' dtype)."""
    n = int(load_library().bc_gated_scan_states_bytes(N, T, C, layout))
    if n == 0:
        raise BoxConvError("gated_scan_states: BC_ERR_SHAPE")
    return torch.empty(n // 4, dtype=torch.float32, device=device)


def gated_scan_fwd(gate: torch.Tensor, x: torch.Tensor, y: torch.Tensor, h0: torch.Tensor | None = None,
                   h_last: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                   states: torch.Tensor | None = None, form: int = BC_GATE_LOGIT, layout: int = BC_TOKENS,
                   ws: torch.Tensor | None = None):
    """gate, x [N, T, C] (BC_TOKENS) or [N, C, T] (BC_MAPS), contiguous in the
    last dimension and of the same strides -> y, dense, of the same shape."""
    what = "gated_scan_fwd"
    N, T, C = _seq_sizes(x, layout, what)
    if gate is None or y is None:
        raise BoxConvError(f"{what}: gate and y must be tensors")
    _need(gate, x.shape, x.dtype, what, "gate")
    _need(y, x.shape, _out_types(x.dtype), what, "y")
    _need(h0, (N, C), _F32, what, "h0")
    _need(h_last, (N, C), _F32, what, "h_last")
    _need(lengths, (N,), torch.int32, what, "lengths")
    lib = load_library()
    if states is not None:
        _need_numel(states, lib.bc_gated_scan_states_bytes(N, T, C, layout) // 4, _F32, what, "states")
    bs, rs = _rows(gate, what, "gate")
    if (bs, rs) != _rows(x, what, "x"):
        raise BoxConvError(f"{what}: gate and x must have the same strides")
    dt = _CODES[x.dtype]
    if ws is None:
        ws = _workspace(lib.bc_gated_scan_workspace_bytes(0, N, T, C, dt, layout), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib.gated_scan_fwd(_data(gate), _data(x), dt, bs, rs, _ptr(h0), _ptr(lengths), _ptr(y), dtype_code(y), _ptr(h_last),
                              _ptr(states), N, T, C, form, layout, _ptr(ws), nbytes, _stream()), what)
    return y


def gated_scan_bwd(gate: torch.Tensor, x: torch.Tensor, states: torch.Tensor, grad_y: torch.Tensor,
                   grad_gate: torch.Tensor, grad_x: torch.Tensor, grad_h_last: torch.Tensor | None = None,
                   grad_h0: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                   form: int = BC_GATE_LOGIT, layout: int = BC_TOKENS, ws: torch.Tensor | None = None):
    """The gradients of gated_scan_fwd; states: what that call kept.  grad_gate
    and grad_x share their strides too (halves of one gradient, for one)."""
    what = "gated_scan_bwd"
    N, T, C = _seq_sizes(x, layout, what)
    if any(v is None for v in (gate, states, grad_y, grad_gate, grad_x)):
        raise BoxConvError(f"{what}: gate, states, grad_y, grad_gate and grad_x must be tensors")
    _need(gate, x.shape, x.dtype, what, "gate")
    _need(grad_y, x.shape, x.dtype, what, "grad_y")
    _need(grad_x, x.shape, _out_types(x.dtype), what, "grad_x")
    _need(grad_gate, x.shape, grad_x.dtype, what, "grad_gate")
    _need(grad_h_last, (N, C), _F32, what, "grad_h_last")
    _need(grad_h0, (N, C), _F32, what, "grad_h0")
    _need(lengths, (N,), torch.int32, what, "lengths")
    lib = load_library()
    _need_numel(states, lib.bc_gated_scan_states_bytes(N, T, C, layout) // 4, _F32, what, "states")
    bs, rs = _rows(gate, what, "gate")
    gbs, grs = _rows(grad_gate, what, "grad_gate")
    if (bs, rs) != _rows(x, what, "x") or (gbs, grs) != _rows(grad_x, what, "grad_x"):
        raise BoxConvError(f"{what}: gate and x, and grad_gate and grad_x, must have the same strides")
    dt = _CODES[x.dtype]
    if ws is None:
        ws = _workspace(lib.bc_gated_scan_workspace_bytes(1, N, T, C, dt, layout), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib.gated_scan_bwd(_data(gate), _data(x), dt, bs, rs, _ptr(states), _ptr(lengths), _ptr(grad_y),
                              _ptr(grad_h_last), _data(grad_gate), _data(grad_x), dtype_code(grad_x), gbs, grs,
                              _ptr(grad_h0), N, T, C, form, layout, _ptr(ws), nbytes, _stream()), what)
    return grad_gate, grad_x


def gated_scan_step(gate: torch.Tensor, x: torch.Tensor, state: torch.Tensor, y: torch.Tensor,
                    slots: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                    form: int = BC_GATE_LOGIT):
    """One token of N sequences: gate, x [N, C] (rows of equal stride), state
    [S, C] fp32 (the pool; state_out, default itself, takes the new states),
    slots [N] int32 -> y [N, C]."""
    what = "gated_scan_step"
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or x.dtype not in _FLOATS:
        raise BoxConvError(f"{what}: x must be a 2-D fp32 or bf16 tensor")
    if gate is None or state is None or y is None:
        raise BoxConvError(f"{what}: gate, state and y must be tensors")
    shape, dtype = x.shape, x.dtype
    N, C = shape
    _need(gate, shape, dtype, what, "gate")
    _need(y, shape, dtype, what, "y")
    S = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() == 2 else None
    _need(state, (S, C), _F32, what, "state")
    _need(state_out, (S, C), _F32, what, "state_out")
    _need(slots, (N,), torch.int32, what, "slots")
    gs, xs = gate.stride(), x.stride()
    if N > 1 and gs[0] != xs[0] or C > 1 and (gs[1] != 1 or xs[1] != 1):
        raise BoxConvError(f"{what}: gate and x must be contiguous in their last dimension and of the same strides")
    sp = _ptr(state)
    lib = _lib or load_library()
    st = lib.gated_scan_step(_data(gate), _data(x), _CODES[dtype], xs[0] if N > 1 else C, sp,
                              sp if state_out is None else _ptr(state_out), _ptr(slots), _ptr(y), N, C, S, form,
                              _stream())
    if st:
        _check(st, what)
    return y


def i8_pitch(K: int) -> int:
    """Bytes between rows of K 8-bit codes."""
    return int(load_library().bc_i8_pitch(K))


def mix_i8_workspace_bytes(N, M, K, P, x_dt: int, layout: int = BC_TOKENS) -> int:
    return int(load_library().bc_mix_i8_workspace_bytes(N, M, K, P, x_dt, layout))


def _mix_input(x, layout, what, name):
    """N, K, P and strides of a mix's input: tokens [T, K] or [N, P, K],
    maps [N, K, P] or [N, K, H, W] (contiguous maps)."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _FLOATS:
        raise BoxConvError(f"{what}: {name} must be an fp32 or bf16 tensor")
    if layout == BC_TOKENS:
        if x.dim() == 2:
            P, K = x.shape
            sr, sc = x.stride()
            if sc != 1 and K > 1:
                raise BoxConvError(f"{what}: {name} must be contiguous in its last dimension")
            if P == 1:
                sr = K
            return 1, K, P, sr * P, sr
        if x.dim() != 3:
            raise BoxConvError(f"{what}: {name} must be [T, K] or [N, P, K]")
        N, P, K = x.shape
    elif layout == BC_MAPS:
        if x.dim() == 4:
            # (a dimension of one element may have any stride)
            if x.shape[2] > 1 and x.stride(2) != (x.shape[3] * x.stride(3) if x.shape[3] > 1 else 1):
                raise BoxConvError(f"{what}: {name}'s maps must be contiguous")
            x = x.flatten(2)
        if x.dim() != 3:
            raise BoxConvError(f"{what}: {name} must be [N, K, P] or [N, K, H, W]")
        N, K, P = x.shape
    else:
        raise BoxConvError(f"{what}: unknown layout {layout}")
    return (N, K, P, *_rows(x, what, name))


def quantize_i8(src: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, layout: int = BC_TOKENS):
    """8-bit codes q [rows, i8_pitch(K)] int8 and scales [rows] fp32 of src:
    tokens or weights [rows, K] ([N, P, K]), or maps [N, K, P] (rows = N * P)."""
    what = "quantize_i8"
    N, K, P, bs, rs = _mix_input(src, layout, what, "src")
    if q is None or scale is None:
        raise BoxConvError(f"{what}: q and scale must be tensors")
    lib = load_library()
    _need(q, (N * P, lib.bc_i8_pitch(K)), torch.int8, what, "q")
    _need(scale, (N * P,), _F32, what, "scale")
    _check(lib.quantize_i8(_data(src), dtype_code(src), bs, rs, _ptr(q), _ptr(scale), N, K, P, layout, _stream()),
           what)
    return q, scale


def pointwise_mix_i8(wq: torch.Tensor, w_scale: torch.Tensor, x: torch.Tensor, out: torch.Tensor,
                     layout: int = BC_TOKENS, x_scale: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                     relu: int = 0, ws: torch.Tensor | None = None):
    """The 1x1 mix in 8-bit codes: wq [M, i8_pitch(K)], w_scale [M] (quantize_i8
    of the weights); x: tokens [T, K] or [N, P, K] -> out [..., M], or maps
    [N, K, P] -> out [N, M, P], fp32 or bf16 each; or x codes [rows, i8_pitch(K)]
    with x_scale [rows]."""
    what = "pointwise_mix_i8"
    if not isinstance(out, torch.Tensor) or out.dtype not in _FLOATS:
        raise BoxConvError(f"{what}: out must be an fp32 or bf16 tensor")
    if not isinstance(wq, torch.Tensor) or wq.dtype is not torch.int8 or wq.dim() != 2 or w_scale is None:
        raise BoxConvError(f"{what}: wq must be a 2-D int8 tensor, with w_scale")
    M, pitch = wq.shape
    _need(w_scale, (M,), _F32, what, "w_scale")
    _need(bias, (M,), _F32, what, "bias")
    if isinstance(x, torch.Tensor) and x.dtype is torch.int8:
        _need(x, (None, pitch), torch.int8, what, "x")
        rows, K = x.shape[0], pitch
        if x_scale is None:
            raise BoxConvError(f"{what}: codes need x_scale")
        _need(x_scale, (rows,), _F32, what, "x_scale")
        if layout == BC_TOKENS:
            N, P = 1, rows
        else:
            N = out.shape[0] if out.dim() else 0
            P = rows // max(N, 1)
        if N * P != rows:
            raise BoxConvError(f"{what}: {rows} rows of codes are not {N} maps")
        bs = rs = 0
    else:
        N, K, P, bs, rs = _mix_input(x, layout, what, "x")
    if (K + 127) // 128 * 128 != pitch:   # i8_pitch(K)
        raise BoxConvError(f"{what}: wq has rows of {pitch} codes, expected i8_pitch({K})")
    shape = out.shape
    if layout == BC_TOKENS:
        if len(shape) == 0 or shape[-1] != M or out.numel() != N * P * M:
            raise BoxConvError(f"{what}: out has shape {tuple(shape)}, expected {N * P} tokens of {M}")
    elif len(shape) not in (3, 4) or shape[0] != N or shape[1] != M or out.numel() != N * M * P:
        raise BoxConvError(f"{what}: out has shape {tuple(shape)}, expected {(N, M, P)}")
    lib = _lib or load_library()
    dt = _CODES[x.dtype]
    xp = _ptr(x) if dt == BC_I8 else _data(x)
    if ws is None:
        ws = _workspace(lib.bc_mix_i8_workspace_bytes(N, M, K, P, dt, layout), x.device)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    st = lib.pointwise_mix_i8(_ptr(wq), _ptr(w_scale), xp, dt, bs, rs, _ptr(x_scale), _ptr(bias), _ptr(out),
                              _CODES[out.dtype], N, M, K, P, relu, layout, _ptr(ws), nbytes, _stream())
    if st:
        _check(st, what)
    return out


# ---- linear-attention blocks --------------------------------------------------

def _strides(t: torch.Tensor, what: str, name: str) -> bc_strides:
    """Of a tensor [N, T, H, D] (or [N, H, D], one token) whose last dimension is
    contiguous; strides of dimensions of one element are zero."""
    shape, s = t.shape, t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise BoxConvError(f"{what}: {name} must be contiguous in its last dimension")
    if len(shape) == 3:
        return bc_strides(s[0] if shape[0] > 1 else 0, 0, s[1] if shape[1] > 1 else 0)
    return bc_strides(s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0)


def _gate_strides(t: torch.Tensor) -> bc_strides:
    """Of a gate [N, T, H], [N, H] (one token) or [H] (a decay for each head)."""
    shape, s = t.shape, [a if n > 1 else 0 for n, a in zip(t.shape, t.stride())]
    if len(shape) == 1:
        return bc_strides(0, 0, s[0])
    return bc_strides(s[0], s[1], s[2]) if len(shape) == 3 else bc_strides(s[0], 0, s[1])


def _one_device(what, *tensors):
    """The library launches on the current device's stream."""
    here = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise BoxConvError("tensors must be on the GPU")
        if here is None:
            here = torch.cuda.current_device()
        if t.get_device() != here:
            raise BoxConvError(f"{what}: tensors must be on the current device ({here})")


def _device() -> int:
    try:
        return torch._C._cuda_getDevice()     # (as in _stream)
    except AttributeError:
        return torch.cuda.current_device()


class _Layouts(dict):
    """What calls of one function were found to be, by the types, shapes and strides
    of their tensors and the call's numbers: checked when they are met first, and
    then kept as the structures that the library takes.  Nothing of a tensor's
    memory or contents is kept, and pointers, devices and alignment are looked at in
    every call.  A token's attention costs 7.2 us of host time in place of 13.2 this way,
    a norm of few rows 7.0 in place of 10.1."""

    def put(self, key, value):
        if len(self) >= 512:
            self.clear()
        self[key] = value
        return value


def _layout(tensors):
    """One key for tensors (None for one that is left out); None if some argument is
    no strided tensor, which the checks then refuse by name."""
    try:
        return tuple([None if t is None else (t.dtype, t.shape, t.stride()) for t in tensors])
    except (AttributeError, RuntimeError, TypeError):
        return None


_forward_calls, _backward_calls, _step_calls, _norm_calls, _norm_grad_calls = (_Layouts() for _ in range(5))


def _here(what, tensors):
    """_one_device, for tensors whose layouts are known."""
    here = _device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            _one_device(what, *tensors)


def _dense(what, layout, *tensors):
    if layout is None:
        raise BoxConvError(f"{what}: arguments must be strided tensors")
    if not all(t is None or t.is_contiguous() for t in tensors):
        raise BoxConvError("tensors must be contiguous")


def _int32(what, *sizes):
    if max(sizes) > 2 ** 31 - 1:
        raise BoxConvError(f"{what}: BC_ERR_SHAPE (a size of 2^31 or more)")


def _attention_sizes(q, k, v, gate, y, form, scale, what, tokens, yname="y"):
    """The sizes of a call, its operands' shapes and types checked against them."""
    dims = 4 if tokens else 3
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (y, yname)):
        if not isinstance(t, torch.Tensor) or t.dim() != dims or t.dtype not in _FLOATS:
            raise BoxConvError(f"{what}: {name} must be a {dims}-D fp32 or bf16 tensor")
    dt, lead, H, Dv = y.dtype, tuple(y.shape[:-2]), y.shape[-2], y.shape[-1]
    Dk = q.shape[-1]
    _need(q, (*lead, q.shape[-2], Dk), dt, what, "q")
    _need(k, (*lead, k.shape[-2], Dk), dt, what, "k")
    _need(v, (*lead, v.shape[-2], Dv), dt, what, "v")
    if not isinstance(gate, torch.Tensor) or gate.dtype not in (torch.float32, dt):
        raise BoxConvError(f"{what}: gate must be a tensor, fp32 or of q's type")
    if gate.dim() != 1:
        _need(gate, (*lead, H), gate.dtype, what, "gate")
    else:
        _need(gate, (H,), gate.dtype, what, "gate")
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if t.shape[-2] == 0 or H % t.shape[-2]:
            raise BoxConvError(f"{what}: {name} has {t.shape[-2]} heads, not a divisor of {H}")
    _int32(what, *lead, H, Dk, Dv)
    return bc_attention(lead[0], lead[1] if tokens else 1, H, q.shape[-2], k.shape[-2], v.shape[-2], Dk, Dv, _CODES[dt],
                        _CODES[gate.dtype], form, float(scale))


def linear_attention_workspace_bytes(op: int, N, T, H, Hq, Hk, Hv, Dk, Dv, dt: int) -> int:
    """op: 0 = linear_attention_fwd, 1 = linear_attention_bwd; dt: dtype code of q."""
    a = bc_attention(N, T, H, Hq, Hk, Hv, Dk, Dv, dt, BC_F32, BC_GATE_LOG, 1.0)
    return int(load_library().bc_linear_attention_workspace_bytes(op, ctypes.byref(a)))


def linear_attention_states(N, T, H, Dk, Dv, device="cuda") -> torch.Tensor:
    """The buffer in which linear_attention_fwd keeps what linear_attention_bwd
    starts from (its layout is the library's)."""
    n = int(load_library().bc_linear_attention_states_bytes(N, T, H, Dk, Dv))
    if n == 0:
        raise BoxConvError("linear_attention_states: BC_ERR_SHAPE")
    return torch.empty(n // 4, dtype=torch.float32, device=device)


def linear_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: torch.Tensor, y: torch.Tensor,
                         s0: torch.Tensor | None = None, s_last: torch.Tensor | None = None,
                         lengths: torch.Tensor | None = None, states: torch.Tensor | None = None,
                         form: int = BC_GATE_LOGIT, scale: float = 1.0, ws: torch.Tensor | None = None):
    """q [N, T, Hq, Dk], k [N, T, Hk, Dk], v [N, T, Hv, Dv] and y [N, T, H, Dv],
    contiguous in the last dimension (views of other layouts are taken as they
    are); gate [N, T, H], or [H]: a decay for each head."""
    what = "linear_attention_fwd"
    scale = float(scale)
    tensors = (q, k, v, gate, y, s0, s_last, lengths, states, ws)
    layout = _layout(tensors)
    call = _forward_calls.get((form, scale, layout))
    lib = _lib or load_library()
    if call is None:
        a = _attention_sizes(q, k, v, gate, y, form, scale, what, True)
        cells = (a.N, a.H, a.Dk, a.Dv)
        _need(s0, cells, _F32, what, "s0")
        _need(s_last, cells, _F32, what, "s_last")
        _need(lengths, (a.N,), torch.int32, what, "lengths")
        if states is not None:
            _need_numel(states, lib.bc_linear_attention_states_bytes(a.N, a.T, a.H, a.Dk, a.Dv) // 4, _F32, what, "states")
        strides = [_strides(t, what, n) for t, n in ((q, "q"), (k, "k"), (v, "v"), (y, "y"))]
        _one_device(what, *tensors)
        _dense(what, layout, s0, s_last, lengths, states, ws)
        nbytes = lib.bc_linear_attention_workspace_bytes(0, a) if ws is None else ws.numel() * ws.element_size()
        call = _forward_calls.put((form, scale, layout), (ctypes.byref(a), *strides, _gate_strides(gate), nbytes))
    _here(what, tensors)
    a, sq, sk, sv, sy, sg, nbytes = call
    if ws is None:
        ws = _workspace(nbytes, q.device)
    p0, p_last, pn, ps, pw = [None if t is None else t.data_ptr() for t in (s0, s_last, lengths, states, ws)]
    st = lib.linear_attention_fwd(a, q.data_ptr(), sq, k.data_ptr(), sk, v.data_ptr(), sv, gate.data_ptr(), sg, p0, pn,
                                  y.data_ptr(), sy, p_last, ps, pw, nbytes, _stream())
    if st:
        _check(st, what)
    return y


def linear_attention_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: torch.Tensor, states: torch.Tensor,
                         grad_y: torch.Tensor, grad_q: torch.Tensor, grad_k: torch.Tensor, grad_v: torch.Tensor,
                         grad_gate: torch.Tensor | None = None, grad_s_last: torch.Tensor | None = None,
                         grad_s0: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                         form: int = BC_GATE_LOGIT, scale: float = 1.0, ws: torch.Tensor | None = None):
    """The gradients of linear_attention_fwd; states: what that call kept.
    grad_gate [N, T, H] or None (a gate [H] is not learned here, or its gradient
    is the sum of grad_gate over sequences and tokens)."""
    what = "linear_attention_bwd"
    scale = float(scale)
    tensors = (q, k, v, gate, states, grad_y, grad_q, grad_k, grad_v, grad_gate, grad_s_last, grad_s0, lengths, ws)
    layout = _layout(tensors)
    call = _backward_calls.get((form, scale, layout))
    lib = _lib or load_library()
    if call is None:
        a = _attention_sizes(q, k, v, gate, grad_y, form, scale, what, True, "grad_y")
        grads = ((grad_q, q, "grad_q"), (grad_k, k, "grad_k"), (grad_v, v, "grad_v"))
        for g, t, name in grads:
            if not isinstance(g, torch.Tensor):
                raise BoxConvError(f"{what}: {name} must be a tensor")
            _need(g, tuple(t.shape), t.dtype, what, name)
        _need(grad_gate, (a.N, a.T, a.H), gate.dtype, what, "grad_gate")
        cells = (a.N, a.H, a.Dk, a.Dv)
        _need(grad_s_last, cells, _F32, what, "grad_s_last")
        _need(grad_s0, cells, _F32, what, "grad_s0")
        _need(lengths, (a.N,), torch.int32, what, "lengths")
        if not isinstance(states, torch.Tensor):
            raise BoxConvError(f"{what}: states must be a tensor")
        _need_numel(states, lib.bc_linear_attention_states_bytes(a.N, a.T, a.H, a.Dk, a.Dv) // 4, _F32, what, "states")
        strides = [_strides(t, what, n) for t, n in ((q, "q"), (k, "k"), (v, "v"), (grad_y, "grad_y"))]
        strides += [_gate_strides(gate)] + [_strides(g, what, name) for g, _, name in grads]
        strides += [bc_strides() if grad_gate is None else _gate_strides(grad_gate)]
        _one_device(what, *tensors)
        _dense(what, layout, states, lengths, grad_s_last, grad_s0, ws)
        nbytes = lib.bc_linear_attention_workspace_bytes(1, a) if ws is None else ws.numel() * ws.element_size()
        call = _backward_calls.put((form, scale, layout), (ctypes.byref(a), *strides, nbytes))
    _here(what, tensors)
    a, sq, sk, sv, sy, sg, gq, gk, gv, gg, nbytes = call
    if ws is None:
        ws = _workspace(nbytes, q.device)
    pq, pk, pv, pg, ps, py, pdq, pdk, pdv, pdg, p_last, p0, pn = [None if t is None else t.data_ptr() for t in tensors[:-1]]
    st = lib.linear_attention_bwd(a, pq, sq, pk, sk, pv, sv, pg, sg, ps, pn, py, sy, p_last, pdq, gq, pdk, gk, pdv, gv, pdg,
                                  gg, p0, None if ws is None else ws.data_ptr(), nbytes, _stream())
    if st:
        _check(st, what)
    return grad_q, grad_k, grad_v


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: torch.Tensor, state: torch.Tensor,
                          y: torch.Tensor, slots: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                          form: int = BC_GATE_LOGIT, scale: float = 1.0):
    """One token of N sequences: q [N, Hq, Dk], k [N, Hk, Dk], v [N, Hv, Dv], gate
    [N, H] or [H], state [S, H, Dk, Dv] fp32 (the pool; state_out, default itself,
    takes the new states), slots [N] int32, none named twice -> y [N, H, Dv], dense."""
    what = "linear_attention_step"
    scale = float(scale)
    tensors = (q, k, v, gate, y, state, state_out, slots)
    layout = _layout(tensors)
    call = _step_calls.get((form, scale, layout))
    if call is None:
        a = _attention_sizes(q, k, v, gate, y, form, scale, what, False)
        S = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() == 4 else None
        if S is None:
            raise BoxConvError(f"{what}: state must be a 4-D tensor")
        _int32(what, S)
        _need(state, (S, a.H, a.Dk, a.Dv), _F32, what, "state")
        _need(state_out, (S, a.H, a.Dk, a.Dv), _F32, what, "state_out")
        _need(slots, (a.N,), torch.int32, what, "slots")
        strides = _strides(q, what, "q"), _strides(k, what, "k"), _strides(v, what, "v"), _gate_strides(gate)
        _one_device(what, *tensors)
        _dense(what, layout, state, state_out, slots, y)
        call = _step_calls.put((form, scale, layout), (ctypes.byref(a), *strides, S))
    _here(what, tensors)
    a, sq, sk, sv, sg, S = call
    sp = state.data_ptr()
    st = (_lib or load_library()).linear_attention_step(
        a, q.data_ptr(), sq, k.data_ptr(), sk, v.data_ptr(), sv, gate.data_ptr(), sg, sp,
        sp if state_out is None else state_out.data_ptr(), None if slots is None else slots.data_ptr(), y.data_ptr(), S,
        _stream())
    if st:
        _check(st, what)
    return y


def _norm_rows(t, shape, dtype, what, name):
    """Pointer and row stride of [..., C], its leading dimensions one run of rows."""
    if t is None:
        return None, 0
    _need(t, shape, dtype, what, name)
    if t.dim() != 2:
        try:
            t = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise BoxConvError(f"{what}: {name}'s rows must be equally far apart") from None
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise BoxConvError(f"{what}: {name} must be contiguous in its last dimension")
    return t.data_ptr(), t.stride(0)


def _norm_sizes(z, groups, kind, act, eps, what):
    if not isinstance(z, torch.Tensor) or z.dim() < 2 or z.dtype not in _FLOATS:
        raise BoxConvError(f"{what}: z must be an fp32 or bf16 tensor [..., C]")
    C = z.shape[-1]
    R = z.numel() // max(C, 1)
    _int32(what, R, C)
    return tuple(z.shape), z.dtype, bc_norm(R, C, groups, kind, act, _CODES[z.dtype], eps)


def block_norm_workspace_bytes(R: int, C: int) -> int:
    return int(load_library().bc_block_norm_workspace_bytes(R, C))


def block_norm_fwd(z: torch.Tensor, gate: torch.Tensor | None = None, x: torch.Tensor | None = None,
                   w_post: torch.Tensor | None = None, res_scale: torch.Tensor | None = None,
                   w_pre: torch.Tensor | None = None, r: torch.Tensor | None = None, y: torch.Tensor | None = None,
                   groups: int = 0, kind: int = BC_NORM_RMS, act: int = BC_ACT_SILU, eps: float = 1e-6):
    """z, gate, x and the outputs r and y (either may be None): [..., C], rows
    equally far apart; weights fp32 [C].  p = norm(z) * w_post by groups (0: z),
    r = x + res_scale * p * act(gate), y = norm(r) * w_pre -> (r, y)."""
    what = "block_norm_fwd"
    eps = float(eps)
    tensors = (z, gate, x, w_post, res_scale, w_pre, r, y)
    layout = _layout(tensors)
    call = _norm_calls.get((groups, kind, act, eps, layout))
    if call is None:
        shape, dt, n = _norm_sizes(z, groups, kind, act, eps, what)
        rows = [_norm_rows(t, shape, dt, what, name) for t, name in ((z, "z"), (gate, "gate"), (x, "x"))]
        for t, name in ((w_post, "w_post"), (res_scale, "res_scale"), (w_pre, "w_pre")):
            _need(t, (n.C,), _F32, what, name)
        rows += [_norm_rows(t, shape, dt, what, name) for t, name in ((r, "r"), (y, "y"))]
        _one_device(what, *tensors)
        _dense(what, layout, w_post, res_scale, w_pre)
        call = _norm_calls.put((groups, kind, act, eps, layout), (ctypes.byref(n), *(step for _, step in rows)))
    _here(what, tensors)
    n, sz, sg, sx, sr, sy = call
    pz, pg, px, wp, ws, wn, pr, py = [None if t is None else t.data_ptr() for t in tensors]
    st = (_lib or load_library()).block_norm_fwd(n, pz, sz, pg, sg, px, sx, wp, ws, wn, pr, sr, py, sy, _stream())
    if st:
        _check(st, what)
    return r, y


def block_norm_bwd(z: torch.Tensor, gate: torch.Tensor | None = None, x: torch.Tensor | None = None,
                   w_post: torch.Tensor | None = None, res_scale: torch.Tensor | None = None,
                   w_pre: torch.Tensor | None = None, grad_r: torch.Tensor | None = None,
                   grad_y: torch.Tensor | None = None, grad_z: torch.Tensor | None = None,
                   grad_gate: torch.Tensor | None = None, grad_x: torch.Tensor | None = None,
                   grad_w_post: torch.Tensor | None = None, grad_res_scale: torch.Tensor | None = None,
                   grad_w_pre: torch.Tensor | None = None, groups: int = 0, kind: int = BC_NORM_RMS,
                   act: int = BC_ACT_SILU, eps: float = 1e-6, ws: torch.Tensor | None = None):
    """The gradients of block_norm_fwd of the same arguments, those that are given
    a tensor -> (grad_z, grad_gate, grad_x)."""
    what = "block_norm_bwd"
    eps = float(eps)
    tensors = (z, gate, x, grad_r, grad_y, grad_z, grad_gate, grad_x, w_post, res_scale, w_pre, grad_w_post, grad_res_scale,
               grad_w_pre, ws)
    layout = _layout(tensors)
    call = _norm_grad_calls.get((groups, kind, act, eps, layout))
    lib = _lib or load_library()
    if call is None:
        shape, dt, n = _norm_sizes(z, groups, kind, act, eps, what)
        names = ("z", "gate", "x", "grad_r", "grad_y", "grad_z", "grad_gate", "grad_x")
        steps = [_norm_rows(t, shape, dt, what, name)[1] for t, name in zip(tensors, names)]
        weights = (w_post, res_scale, w_pre, grad_w_post, grad_res_scale, grad_w_pre)
        for t, name in zip(weights, ("w_post", "res_scale", "w_pre", "grad_w_post", "grad_res_scale", "grad_w_pre")):
            _need(t, (n.C,), _F32, what, name)
        _one_device(what, *tensors)
        _dense(what, layout, *weights, ws)
        if ws is not None:
            nbytes = ws.numel() * ws.element_size()
        else:
            nbytes = lib.bc_block_norm_workspace_bytes(n.R, n.C) if any(t is not None for t in weights[3:]) else 0
        call = _norm_grad_calls.put((groups, kind, act, eps, layout), (ctypes.byref(n), *steps, nbytes))
    _here(what, tensors)
    n, sz, sg, sx, sr, sy, sdz, sdg, sdx, nbytes = call
    if ws is None:
        ws = _workspace(nbytes, z.device)
    pz, pg, px, pr, py, pdz, pdg, pdx, *pw = [None if t is None else t.data_ptr() for t in tensors[:-1]]
    st = lib.block_norm_bwd(n, pz, sz, pg, sg, px, sx, *pw[:3], pr, sr, py, sy, pdz, sdz, pdg, sdg, pdx, sdx, *pw[3:],
                            None if ws is None else ws.data_ptr(), nbytes, _stream())
    if st:
        _check(st, what)
    return grad_z, grad_gate, grad_x
