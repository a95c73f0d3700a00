"""Layer operators of denoisers on torch CUDA tensors: layer norm, the gated feed-forward block, the linear layer with its
epilogue, dropout, and the norms around a residual block with its gate, each with its backward pass (include/sds.h documents the formulas). Every call enqueues on the current stream of its
tensors' device and does not wait. Outputs and workspaces are allocated by torch unless they are passed in. A bad
argument raises ValueError, an error of the library SdsError. Nothing is recorded for autograd: the backward calls are
the gradients. A forward call whose inputs require gradients (or carry forward-mode tangents) outside torch.no_grad()
warns of that.
"""
from __future__ import annotations

import ctypes as C

from . import binding as sb

ACTIVATIONS = sb.ACTIVATIONS

_native = None       # the extension that checks arguments, allocates and calls libsds (csrc/sds_torch.cpp)


def _ext():
    """The extension, built first if its source is newer (or it was built for another torch); a call on tensors needs it."""
    global _native
    if _native is None:
        import importlib.machinery
        import importlib.util
        import torch  # noqa: F401  (the extension's libraries)
        from . import build
        sb.load()
        if build.needs_ext_build():
            build.build_ext()
        name, path = __package__ + "._sds_torch", build.ext_path()
        loader = importlib.machinery.ExtensionFileLoader(name, path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location(name, path, loader=loader))
        loader.exec_module(module)
        _native = module
    return _native


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, *, out_dtype=None, stats: bool = False, out=None):
    """sds_layer_norm over the last dimension of x (float32, bfloat16 or float16; leading dimensions that make evenly
    spaced rows, which do not overlap). weight, bias: vectors of one type, or None. out_dtype: x's type (default), or for float x any of the
    three. Returns y, with stats=True (y, mean, rstd): the float row statistics that layer_norm_backward takes."""
    return (_native or _ext()).layer_norm(x, weight, bias, eps, out_dtype, stats, out)


def layer_norm_backward(dy, x, weight, mean, rstd, *, want=(True, True, True), workspace=None):
    """sds_layer_norm_backward: (dx, dweight, dbias) from dy (of the forward output's type) and the forward call's x,
    weight (or None) and row statistics. want: which of the three to compute (None is returned for the
    others). The weights' gradients have weight's type, float32 without one."""
    return (_native or _ext()).layer_norm_backward(dy, x, weight, mean, rstd, want, workspace)


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------


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
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    return (_native or _ext()).gated_ffn(x, w_gate, w_up, w_down, act, keep, out, workspace)


def gated_ffn_backward(dy, x, w_gate, w_up, w_down, kept, *, want=(True, True, True, True), workspace=None):
    """sds_gated_ffn_backward: (dx, dw_gate, dw_up, dw_down) from dy and the forward call's x, weights and kept.
    want: which of the four to compute (None is returned for the others)."""
    return (_native or _ext()).gated_ffn_backward(dy, x, w_gate, w_up, w_down, kept, want, workspace)


def _wait_status(name: str, workspace) -> None:
    """Waits for the current stream and raises if a bounded wait gave up: name_status of a workspace, or name_gave_up."""
    import torch
    if workspace is None:
        where, args, device = name + "_gave_up", (), None
    else:
        where, args, device = name + "_status", (workspace.data_ptr(),), workspace.device
    with torch.cuda.device(device):
        rc = getattr(sb.load(), where)(*args, torch.cuda.current_stream().cuda_stream)
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, where)


def gated_ffn_status(workspace=None) -> None:
    """Waits for the current stream and raises if a bounded wait of the last gated_ffn call (or its backward) that
    was given this workspace gave up. Without one: if a wait of any such call on the current device did since this was asked
    last, whatever its workspace (those that the calls allocate themselves have no other report)."""
    _wait_status("sds_gated_ffn", workspace)


# ---------------------------------------------------------------------------------------------
# linear layer
# ---------------------------------------------------------------------------------------------


def _activation(name) -> int:
    act = sb.SDS_ACT_NONE if name is None else ACTIVATIONS.get(name)
    if act is None:
        raise ValueError(f"activation must be None or one of {sorted(ACTIVATIONS)}")
    return act


def linear(x, weight, bias=None, activation=None, *, table=None, step=None, residual=None, out_dtype=None, keep: bool = False,
           out=None, workspace=None):
    """sds_linear: y = act(x W^T + bias + table[step]) + residual for x [..., k] and weight [n, k] (bfloat16 or float16, k a
    multiple of 8); bias [n] of any of the three types; table [steps, n] of x's type with step, int32, one row of the table per
    row of x (a row whose step is outside the table becomes NaN); residual [..., n] of the output's type. activation None,
    "silu", "gelu" or "gelu_tanh". out_dtype: x's type (default) or float32. With keep=True returns (y, kept) with what
    linear_backward needs."""
    return (_native or _ext()).linear(x, weight, bias, _activation(activation), table, step, residual, out_dtype, keep, out, workspace)


def linear_backward(dy, x, weight, kept, *, bias=None, table=None, step=None, want=(True, True, True, True), workspace=None):
    """sds_linear_backward: (dx, dweight, dbias, dtable) from dy (of the forward output's type) and the forward call's x,
    weight, kept, bias, table and step (of bias and table only size and type count). want: which of the four to compute; None
    is returned for the others, and for the bias and the table where there was none. The residual's gradient is dy. A row whose step is
    outside the table takes no part: zeros in dx, nothing in the others."""
    return (_native or _ext()).linear_backward(dy, x, weight, kept, bias, table, step, want, workspace)


def linear_status(workspace=None) -> None:
    """gated_ffn_status for linear and linear_backward."""
    _wait_status("sds_linear", workspace)


# ---------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------


def dropout(x, p: float, seed: int, step=0, *, residual=None, row0: int = 0, out=None):
    """sds_dropout: D x + residual with D = 0 or 1 / (1 - p) (p rounded to a multiple of 2^-16), drawn from (seed, step, row,
    column) and never stored. step: the training step, a number or an int32 CUDA tensor of one element (read when the kernel
    runs: a captured graph draws anew); row0: global number of x's first row. The output has the residual's type, x's without one."""
    return (_native or _ext()).dropout(x, p, seed, step, row0, residual, None, out)


def dropout_backward(dy, p: float, seed: int, step=0, *, row0: int = 0, out_dtype=None, out=None):
    """The gradient of dropout's x: D dy with the forward call's p, seed, step and row0. out_dtype: x's type, where it is not
    dy's. The residual's gradient is dy."""
    return (_native or _ext()).dropout(dy, p, seed, step, row0, None, out_dtype, out)


# ---------------------------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------------------------

NORMS = ("layer", "rms")


def _rms(kind: str) -> bool:
    if kind not in NORMS:
        raise ValueError(f"kind must be one of {NORMS}")
    return kind == "rms"


def residual_norm(r, h=None, *, weight=None, bias=None, scale=None, shift=None, gate=None, post: bool = False, post_weight=None,
                  kind: str = "layer", alpha: float = 1.0, eps: float = 1e-5, p: float = 0.0, seed: int = 0, step=0, row0: int = 0,
                  out_dtype=None, keep: bool = False, out=None, stream_out=None):
    """sds_residual_norm: from one residual block to the next. For the stream r [..., d] and the block's output h:
    q = post_weight * norm(h) with post=True, else h;  stream = r + alpha gate dropout(q);  n = (norm(stream) weight + bias) (1 + scale) + shift.
    kind "layer" or "rms" (both norms); gate, scale and shift [groups, d] (slices of one tensor will do), each row of them for
    rows / groups consecutive rows of r; p, seed, step and row0 as for dropout. Without h there is no block behind: n is that of r. n has
    h's type (out_dtype without h): r's, or for a float r any of the three. Returns (stream, n), with keep=True
    (stream, n, kept) with what residual_norm_backward needs; without h the stream is r itself."""
    return (_native or _ext()).residual_norm(r, h, weight, bias, scale, shift, gate, post, post_weight, _rms(kind), alpha, eps, p, seed,
                                             step, row0, out_dtype, keep, out, stream_out)


def residual_norm_backward(dn, dr, r, h, kept, *, weight=None, bias=None, scale=None, shift=None, gate=None, post: bool = False,
                           post_weight=None, kind: str = "layer", alpha: float = 1.0, p: float = 0.0, seed: int = 0, step=0,
                           row0: int = 0, want=(True,) * 8, workspace=None):
    """sds_residual_norm_backward: (dr, dh, dweight, dbias, dscale, dshift, dgate, dpost_weight) from dn, the stream's own gradient dr
    (None = zeros) and the forward call's arguments. want: which of the eight to compute; None is returned for the others and
    for what there was not."""
    return (_native or _ext()).residual_norm_backward(dn, dr, r, h, kept, weight, bias, scale, shift, gate, post, post_weight, _rms(kind),
                                                      alpha, 0.0, p, seed, step, row0, want, workspace)
