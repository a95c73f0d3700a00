"""Layer operators of gated denoisers on torch CUDA tensors: layer norm and the gated feed-forward block, each
with its backward pass. Argument checks and marshalling only; the work is in libsds (include/sds.h documents the
formulas). Every call enqueues on the current stream of its tensors' device and does not wait. Outputs and
workspaces are allocated by torch unless they are passed in.

Small calls take a few microseconds on the GPU, so the way to the launch is kept short: contiguous tensors are
recognised by one test, devices are compared by index, sizes that depend on the shapes alone are computed once.
"""
from __future__ import annotations

import ctypes as C
import functools

from . import binding as sb

ACTIVATIONS = sb.ACTIVATIONS

_torch = None        # set by _load
_lib = None
_code = {}           # torch dtype -> SDS_F32, SDS_BF16, SDS_F16
_raw_stream = None   # device index -> cudaStream_t of its current stream


def _load():
    global _torch, _lib, _raw_stream
    import torch
    # torch's own short way to the handle; a Stream object per call costs three microseconds
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        _raw_stream = lambda dev: torch.cuda.current_stream(dev).cuda_stream  # noqa: E731
    _code.update({torch.float32: sb.SDS_F32, torch.bfloat16: sb.SDS_BF16, torch.float16: sb.SDS_F16})
    _torch = torch
    _lib = sb.load()


def _dtype(x) -> int:
    code = _code.get(x)
    if code is None:
        raise ValueError(f"unsupported dtype {x}")
    return code


def _rows(x, what: str):
    """(rows, d, elements between rows) of a CUDA tensor [..., d] whose leading dimensions make evenly spaced rows."""
    if not x.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    shape = x.shape
    if len(shape) < 1 or shape[-1] < 1:
        raise ValueError(f"{what} must be [..., d], got {tuple(shape)}")
    d = shape[-1]
    rows = x.numel() // d
    if x.is_contiguous() or rows == 0:
        return rows, d, d
    if d > 1 and x.stride(-1) != 1:
        raise ValueError(f"{what} must be contiguous along its last dimension")
    ld, span = None, 1                           # span: rows covered by the dimensions seen so far, innermost first
    for k in range(x.dim() - 2, -1, -1):
        if shape[k] == 1:
            continue
        if ld is None:
            ld = x.stride(k)
        elif x.stride(k) != ld * span:
            raise ValueError(f"{what}: the leading dimensions must be evenly spaced rows")
        span *= shape[k]
    return rows, d, (d if ld is None else ld)


def _vector(v, d: int, dev: int, what: str) -> int:
    """Pointer of a contiguous vector of d elements on device index dev."""
    if v.dim() != 1 or v.numel() != d or not v.is_contiguous() or v.get_device() != dev:
        raise ValueError(f"{what} must be a contiguous vector of {d} on x's device, got {tuple(v.shape)} on {v.device}")
    return v.data_ptr()


def _out(out, like, dtype, dev: int):
    if tuple(out.shape) != tuple(like.shape) or out.dtype != dtype or out.get_device() != dev:
        raise ValueError(f"out must be a {dtype} tensor of shape {tuple(like.shape)} on {like.device}")
    return _rows(out, "out")[2]


def _call(fn, dev: int, *args):
    """fn(*args, stream) with dev as the current device, on its current stream."""
    if _torch.cuda.current_device() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with _torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, fn.__name__)


def _workspace(ws, need: int, x, dev: int):
    if ws is None:
        return x.new_empty(need, dtype=_torch.uint8)
    if ws.dtype != _torch.uint8 or ws.get_device() != dev or not ws.is_contiguous() or ws.numel() < need:
        raise ValueError(f"workspace must be a contiguous uint8 tensor of at least {need} bytes on x's device")
    return ws


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, *, out_dtype=None, stats: bool = False, out=None):
    """sds_layer_norm over the last dimension of x (float32, bfloat16 or float16). weight, bias: vectors of one type,
    or None. out_dtype: x's type (default), or for float x any of the three. Returns y, with stats=True
    (y, mean, rstd): the float row statistics that layer_norm_backward takes."""
    if _lib is None:
        _load()
    rows, d, ldx = _rows(x, "x")
    dev = x.get_device()
    tx = tw = _dtype(x.dtype)
    wp = bp = None
    if weight is not None:
        wp, tw = _vector(weight, d, dev, "weight"), _dtype(weight.dtype)
        if bias is not None and bias.dtype != weight.dtype:
            raise ValueError("weight and bias must have the same type")
    if bias is not None:
        bp, tw = _vector(bias, d, dev, "bias"), _dtype(bias.dtype)
    if out_dtype is None:
        out_dtype = x.dtype
    if out is None:
        y, ldy = x.new_empty(x.shape, dtype=out_dtype), d
    else:
        y, ldy = out, _out(out, x, out_dtype, dev)
    if not stats:
        _call(_lib.sds_layer_norm, dev, x.data_ptr(), ldx, tx, wp, bp, tw, rows, d, eps, y.data_ptr(), ldy,
              _dtype(out_dtype), None, None)
        return y
    mean = x.new_empty(x.shape[:-1], dtype=_torch.float32)
    rstd = _torch.empty_like(mean)
    _call(_lib.sds_layer_norm, dev, x.data_ptr(), ldx, tx, wp, bp, tw, rows, d, eps, y.data_ptr(), ldy, _dtype(out_dtype),
          mean.data_ptr(), rstd.data_ptr())
    return y, mean, rstd


@functools.lru_cache(maxsize=1024)
def _norm_workspace_bytes(rows: int, d: int) -> int:
    need = C.c_size_t(0)
    rc = _lib.sds_layer_norm_workspace_bytes(rows, d, C.byref(need))
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, "sds_layer_norm_workspace_bytes")
    return need.value


def layer_norm_backward(dy, x, weight, mean, rstd, *, want=(True, True, True), workspace=None):
    """sds_layer_norm_backward: (dx, dweight, dbias) from dy (of the forward output's type) and the forward call's x,
    weight (or None) and row statistics. want: which of the three to compute (None is returned for the
    others). The weights' gradients have weight's type, float32 without one."""
    if _lib is None:
        _load()
    rows, d, ldx = _rows(x, "x")
    dev = x.get_device()
    if dy.shape != x.shape or dy.get_device() != dev:
        raise ValueError(f"dy must have x's shape {tuple(x.shape)} and device")
    lddy = _rows(dy, "dy")[2]
    wt = _torch.float32
    wp = None
    if weight is not None:
        wp, wt = _vector(weight, d, dev, "weight"), weight.dtype
    for v in (mean, rstd):
        if v.dtype != _torch.float32 or v.numel() != rows or not v.is_contiguous() or v.get_device() != dev:
            raise ValueError("mean and rstd must be contiguous float32 tensors with one value per row, on x's device")
    dx = x.new_empty(x.shape) if want[0] else None
    dw = x.new_empty(d, dtype=wt) if want[1] else None
    db = x.new_empty(d, dtype=wt) if want[2] else None
    ws = _workspace(workspace, _norm_workspace_bytes(rows, d), x, dev)
    _call(_lib.sds_layer_norm_backward, dev, dy.data_ptr(), lddy, _dtype(dy.dtype), x.data_ptr(), ldx, _dtype(x.dtype), wp,
          _dtype(wt), mean.data_ptr(), rstd.data_ptr(), rows, d, dx.data_ptr() if want[0] else None, d,
          dw.data_ptr() if want[1] else None, db.data_ptr() if want[2] else None, ws.data_ptr(), ws.numel())
    return dx, dw, db


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------


def _ffn_shapes(x, w_gate, w_up, w_down):
    rows, d, ldx = _rows(x, "x")
    dev, dtype = x.get_device(), x.dtype
    f = w_gate.shape[0] if w_gate.dim() == 2 else -1
    if w_gate.shape != (f, d) or w_up.shape != (f, d) or w_down.shape != (d, f):
        raise ValueError(f"w_gate and w_up must be [f, {d}] and w_down [{d}, f], got {tuple(w_gate.shape)}, "
                         f"{tuple(w_up.shape)} and {tuple(w_down.shape)}")
    for w in (w_gate, w_up, w_down):
        if w.dtype != dtype or w.get_device() != dev or not w.is_contiguous():
            raise ValueError(f"the weights must be contiguous {dtype} tensors on x's device")
    return rows, d, ldx, f, dev


@functools.lru_cache(maxsize=1024)
def gated_ffn_bytes(rows: int, d: int, f: int):
    """sds_gated_ffn_bytes: a structure with keep_bytes, forward_bytes, forward_keep_bytes and backward_bytes."""
    s = sb.SdsGatedFfnSizes()
    rc = sb.load().sds_gated_ffn_bytes(rows, d, f, C.byref(s))
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, "sds_gated_ffn_bytes")
    return s


def gated_ffn(x, w_gate, w_up, w_down, activation: str = "silu", *, keep: bool = False, out=None, workspace=None):
    """sds_gated_ffn: y = (act(x Wg^T) * (x Wu^T)) Wd^T for x [..., d] (bfloat16 or float16), w_gate and w_up [f, d],
    w_down [d, f]; activation "silu", "gelu" or "gelu_tanh". With keep=True returns (y, kept) with what
    gated_ffn_backward needs."""
    if _lib is None:
        _load()
    rows, d, ldx, f, dev = _ffn_shapes(x, w_gate, w_up, w_down)
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    s = gated_ffn_bytes(rows, d, f)
    if out is None:
        y, ldy = x.new_empty(x.shape), d
    else:
        y, ldy = out, _out(out, x, x.dtype, dev)
    kept = x.new_empty(s.keep_bytes, dtype=_torch.uint8) if keep else None
    ws = _workspace(workspace, s.forward_keep_bytes if keep else s.forward_bytes, x, dev)
    _call(_lib.sds_gated_ffn, dev, x.data_ptr(), ldx, _dtype(x.dtype), rows, d, f, w_gate.data_ptr(), w_up.data_ptr(),
          w_down.data_ptr(), act, y.data_ptr(), ldy, kept.data_ptr() if keep else None, ws.data_ptr(), ws.numel())
    return (y, kept) if keep else y


def gated_ffn_backward(dy, x, w_gate, w_up, w_down, kept, *, want=(True, True, True, True), workspace=None):
    """sds_gated_ffn_backward: (dx, dw_gate, dw_up, dw_down) from dy and the forward call's x, weights and kept.
    want: which of the four to compute (None is returned for the others)."""
    if _lib is None:
        _load()
    rows, d, ldx, f, dev = _ffn_shapes(x, w_gate, w_up, w_down)
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.get_device() != dev:
        raise ValueError(f"dy must have x's shape {tuple(x.shape)}, type {x.dtype} and device")
    lddy = _rows(dy, "dy")[2]
    s = gated_ffn_bytes(rows, d, f)
    if (kept.dtype != _torch.uint8 or not kept.is_contiguous() or kept.numel() < s.keep_bytes
            or kept.get_device() != dev):
        raise ValueError("kept must be what gated_ffn(keep=True) returned for these sizes")
    grads = [x.new_empty(v.shape) if w else None
             for w, v in zip(want, (x, w_gate, w_up, w_down))]
    dx, dwg, dwu, dwd = (None if g is None else g.data_ptr() for g in grads)
    ws = _workspace(workspace, s.backward_bytes, x, dev)
    _call(_lib.sds_gated_ffn_backward, dev, dy.data_ptr(), lddy, x.data_ptr(), ldx, _dtype(x.dtype), rows, d, f,
          w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), kept.data_ptr(), dx, d, dwg, dwu, dwd, ws.data_ptr(),
          ws.numel())
    return tuple(grads)


def gated_ffn_status(workspace) -> None:
    """Waits for the current stream and raises if a bounded wait of the last gated_ffn call (or its backward) that
    was given this workspace gave up."""
    if _lib is None:
        _load()
    _call(_lib.sds_gated_ffn_status, workspace.get_device(), workspace.data_ptr())
