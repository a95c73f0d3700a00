"""Layer operators of gated denoisers on torch CUDA tensors: layer norm and the gated feed-forward block, each
with its backward pass. Argument checks and marshalling only; the work is in libsds (include/sds.h documents the
formulas). Every call enqueues on the current stream of its tensors' device and does not wait. Outputs and
workspaces are allocated by torch unless they are passed in.
"""
from __future__ import annotations

import ctypes as C

from . import binding as sb

ACTIVATIONS = {"silu": sb.SDS_ACT_SILU, "gelu": sb.SDS_ACT_GELU, "gelu_tanh": sb.SDS_ACT_GELU_TANH}


def _torch():
    import torch
    return torch


def _dtype(t, x) -> int:
    code = {t.float32: sb.SDS_F32, t.bfloat16: sb.SDS_BF16, t.float16: sb.SDS_F16}.get(x)
    if code is None:
        raise ValueError(f"unsupported dtype {x}")
    return code


def _rows(x, what: str, d=None):
    """(rows, d, elements between rows) of a tensor [..., d] whose leading dimensions make evenly spaced rows."""
    if not x.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if x.dim() < 1 or x.shape[-1] < 1 or (d is not None and x.shape[-1] != d):
        raise ValueError(f"{what} must be [..., {d if d is not None else 'd'}], got {tuple(x.shape)}")
    n = x.shape[-1]
    rows = x.numel() // n
    if rows == 0:
        return 0, n, n
    if n > 1 and x.stride(-1) != 1:
        raise ValueError(f"{what} must be contiguous along its last dimension")
    ld = None
    span = 1                                     # rows covered by the dimensions seen so far, innermost first
    for k in range(x.dim() - 2, -1, -1):
        if x.shape[k] == 1:
            continue
        if ld is None:
            ld = x.stride(k)
        elif x.stride(k) != ld * span:
            raise ValueError(f"{what}: the leading dimensions must be evenly spaced rows")
        span *= x.shape[k]
    return rows, n, (n if ld is None else ld)


def _same_device(x, **others):
    for name, v in others.items():
        if v is not None and v.device != x.device:
            raise ValueError(f"{name} is on {v.device}, not on {x.device}")


def _vector(v, d: int, what: str):
    if v is not None and (tuple(v.shape) != (d,) or not v.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous vector of {d}, got {tuple(v.shape)}")


def _out(out, like_shape, dtype, device, what: str):
    t = _torch()
    if out is None:
        return t.empty(like_shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(like_shape) or out.dtype != dtype or out.device != device:
        raise ValueError(f"{what} must be a {dtype} tensor of shape {tuple(like_shape)} on {device}")
    return out


class _On:
    """Makes a device current for a launch where it is not already."""

    def __init__(self, device):
        t = _torch()
        self.guard = None if t.cuda.current_device() == device.index else t.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()

    def __exit__(self, *a):
        if self.guard is not None:
            self.guard.__exit__(*a)


def _stream(x) -> int:
    return _torch().cuda.current_stream(x.device).cuda_stream


def _ptr(x):
    return None if x is None else x.data_ptr()


def _check(rc: int, where: str):
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, where)


def _workspace(ws, need: int, device, what: str):
    t = _torch()
    if ws is None:
        return t.empty(need, dtype=t.uint8, device=device)
    if ws.dtype != t.uint8 or ws.device != device or not ws.is_contiguous() or ws.numel() < need:
        raise ValueError(f"{what} must be a contiguous uint8 tensor of at least {need} bytes on {device}")
    return ws


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, *, out_dtype=None, stats: bool = False, out=None):
    """sds_layer_norm over the last dimension of x (float32, bfloat16 or float16). weight, bias: vectors of one type,
    or None. out_dtype: x's type (default), or for float x any of the three. Returns y, with stats=True
    (y, mean, rstd): the float row statistics that layer_norm_backward takes."""
    t = _torch()
    rows, d, ldx = _rows(x, "x")
    _vector(weight, d, "weight")
    _vector(bias, d, "bias")
    _same_device(x, weight=weight, bias=bias)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have the same type")
    y = _out(out, x.shape, out_dtype or x.dtype, x.device, "out")
    _, _, ldy = _rows(y, "out")
    wt = weight if weight is not None else bias
    mean = rstd = None
    if stats:
        mean = t.empty(x.shape[:-1], dtype=t.float32, device=x.device)
        rstd = t.empty(x.shape[:-1], dtype=t.float32, device=x.device)
    with _On(x.device):
        _check(sb.load().sds_layer_norm(x.data_ptr(), ldx, _dtype(t, x.dtype), _ptr(weight), _ptr(bias),
                                        sb.SDS_F32 if wt is None else _dtype(t, wt.dtype), rows, d, eps, y.data_ptr(),
                                        ldy, _dtype(t, y.dtype), _ptr(mean), _ptr(rstd), _stream(x)), "sds_layer_norm")
    return (y, mean, rstd) if stats else y


def layer_norm_backward(dy, x, weight, mean, rstd, *, want=(True, True, True), workspace=None):
    """sds_layer_norm_backward: (dx, dweight, dbias) from dy (of the forward output's type) and the forward call's x,
    weight (or None) and row statistics. want: which of the three to compute (None is returned for the
    others). The weights' gradients have weight's type, float32 without one."""
    t = _torch()
    rows, d, ldx = _rows(x, "x")
    rows_y, _, lddy = _rows(dy, "dy", d)
    if tuple(dy.shape) != tuple(x.shape):
        raise ValueError(f"dy must have x's shape {tuple(x.shape)}, got {tuple(dy.shape)}")
    _vector(weight, d, "weight")
    for name, v in (("mean", mean), ("rstd", rstd)):
        if v.dtype != t.float32 or not v.is_contiguous() or v.numel() != rows:
            raise ValueError(f"{name} must be a contiguous float32 tensor with one value per row")
    _same_device(x, dy=dy, weight=weight, mean=mean, rstd=rstd)
    wt = t.float32 if weight is None else weight.dtype
    dx = t.empty(x.shape, dtype=x.dtype, device=x.device) if want[0] else None
    dw = t.empty(d, dtype=wt, device=x.device) if want[1] else None
    db = t.empty(d, dtype=wt, device=x.device) if want[2] else None
    lib = sb.load()
    need = C.c_size_t(0)
    _check(lib.sds_layer_norm_workspace_bytes(rows, d, C.byref(need)), "sds_layer_norm_workspace_bytes")
    ws = _workspace(workspace, need.value, x.device, "workspace")
    with _On(x.device):
        _check(lib.sds_layer_norm_backward(dy.data_ptr(), lddy, _dtype(t, dy.dtype), x.data_ptr(), ldx,
                                           _dtype(t, x.dtype), _ptr(weight), _dtype(t, wt), mean.data_ptr(),
                                           rstd.data_ptr(), rows, d, _ptr(dx), d, _ptr(dw), _ptr(db), ws.data_ptr(),
                                           ws.numel(), _stream(x)), "sds_layer_norm_backward")
    return dx, dw, db


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------


def _ffn_shapes(x, w_gate, w_up, w_down):
    rows, d, ldx = _rows(x, "x")
    f = w_gate.shape[0] if w_gate.dim() == 2 else -1
    for name, w, shape in (("w_gate", w_gate, (f, d)), ("w_up", w_up, (f, d)), ("w_down", w_down, (d, f))):
        if tuple(w.shape) != shape or not w.is_contiguous():
            raise ValueError(f"{name} must be contiguous {shape}, got {tuple(w.shape)}")
        if w.dtype != x.dtype:
            raise ValueError(f"{name} must have x's type {x.dtype}")
    _same_device(x, w_gate=w_gate, w_up=w_up, w_down=w_down)
    return rows, d, ldx, f


def gated_ffn_bytes(rows: int, d: int, f: int):
    """sds_gated_ffn_bytes: a structure with keep_bytes, forward_bytes, forward_keep_bytes and backward_bytes."""
    s = sb.SdsGatedFfnSizes()
    _check(sb.load().sds_gated_ffn_bytes(rows, d, f, C.byref(s)), "sds_gated_ffn_bytes")
    return s


def gated_ffn(x, w_gate, w_up, w_down, activation: str = "silu", *, keep: bool = False, out=None, workspace=None):
    """sds_gated_ffn: y = (act(x Wg^T) * (x Wu^T)) Wd^T for x [..., d] (bfloat16 or float16), w_gate and w_up [f, d],
    w_down [d, f]; activation "silu", "gelu" or "gelu_tanh". With keep=True returns (y, kept) with what
    gated_ffn_backward needs."""
    t = _torch()
    rows, d, ldx, f = _ffn_shapes(x, w_gate, w_up, w_down)
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _, _, ldy = _rows(y, "out")
    s = gated_ffn_bytes(rows, d, f)
    kept = t.empty(s.keep_bytes, dtype=t.uint8, device=x.device) if keep else None
    ws = _workspace(workspace, s.forward_keep_bytes if keep else s.forward_bytes, x.device, "workspace")
    with _On(x.device):
        _check(sb.load().sds_gated_ffn(x.data_ptr(), ldx, _dtype(t, x.dtype), rows, d, f, w_gate.data_ptr(),
                                       w_up.data_ptr(), w_down.data_ptr(), ACTIVATIONS[activation], y.data_ptr(), ldy,
                                       _ptr(kept), ws.data_ptr(), ws.numel(), _stream(x)), "sds_gated_ffn")
    return (y, kept) if keep else y


def gated_ffn_backward(dy, x, w_gate, w_up, w_down, kept, *, want=(True, True, True, True), workspace=None):
    """sds_gated_ffn_backward: (dx, dw_gate, dw_up, dw_down) from dy and the forward call's x, weights and kept.
    want: which of the four to compute (None is returned for the others)."""
    t = _torch()
    rows, d, ldx, f = _ffn_shapes(x, w_gate, w_up, w_down)
    if tuple(dy.shape) != tuple(x.shape) or dy.dtype != x.dtype:
        raise ValueError(f"dy must have x's shape {tuple(x.shape)} and type {x.dtype}")
    _, _, lddy = _rows(dy, "dy", d)
    s = gated_ffn_bytes(rows, d, f)
    if kept.dtype != t.uint8 or not kept.is_contiguous() or kept.numel() < s.keep_bytes:
        raise ValueError("kept must be what gated_ffn(keep=True) returned for these sizes")
    _same_device(x, dy=dy, kept=kept)
    new = lambda w, like: t.empty(like.shape, dtype=x.dtype, device=x.device) if w else None  # noqa: E731
    dx, dwg, dwu, dwd = (new(w, like) for w, like in zip(want, (x, w_gate, w_up, w_down)))
    ws = _workspace(workspace, s.backward_bytes, x.device, "workspace")
    with _On(x.device):
        _check(sb.load().sds_gated_ffn_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, _dtype(t, x.dtype), rows, d, f,
                                                w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
                                                kept.data_ptr(), _ptr(dx), d, _ptr(dwg), _ptr(dwu), _ptr(dwd),
                                                ws.data_ptr(), ws.numel(), _stream(x)), "sds_gated_ffn_backward")
    return dx, dwg, dwu, dwd


def gated_ffn_status(workspace) -> None:
    """Waits for the current stream and raises if a bounded wait of the last gated_ffn call (or its backward) that
    was given this workspace gave up."""
    with _On(workspace.device):
        _check(sb.load().sds_gated_ffn_status(workspace.data_ptr(), _stream(workspace)), "sds_gated_ffn_status")
