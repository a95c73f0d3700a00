"""Layer operators of gated denoisers on torch CUDA tensors: layer norm and the gated feed-forward block, each
with its backward pass (include/sds.h documents the formulas). Every call enqueues on the current stream of its
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


def gated_ffn_status(workspace=None) -> None:
    """Waits for the current stream and raises if a bounded wait of the last gated_ffn call (or its backward) that
    was given this workspace gave up. Without one: if a wait of any such call on the current device did since this was asked
    last, whatever its workspace (those that the calls allocate themselves have no other report)."""
    import torch
    if workspace is None:
        where, rc = "sds_gated_ffn_gave_up", sb.load().sds_gated_ffn_gave_up(torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(workspace.device):
            where, rc = "sds_gated_ffn_status", sb.load().sds_gated_ffn_status(workspace.data_ptr(), torch.cuda.current_stream().cuda_stream)
    if rc != sb.SDS_OK:
        raise sb.SdsError(rc, where)
