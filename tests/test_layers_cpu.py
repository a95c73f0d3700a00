"""Refusals of the layer operators' C entry points: every bad argument is answered on the host, before any launch
(no GPU is needed; the pointers are numbers that nothing reads)."""
import ctypes as C

import pytest

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb

X, Y, W, B, M, R, WS = (0x10000 * (i + 1) for i in range(7))


def _norm(**kw):
    a = dict(x=X, ldx=64, tx=sb.SDS_F32, w=W, b=B, tw=sb.SDS_F32, rows=4, d=64, eps=1e-5, y=Y, ldy=64, ty=sb.SDS_F32,
             mean=M, rstd=R)
    a.update(kw)
    return sds.load().sds_layer_norm(a["x"], a["ldx"], a["tx"], a["w"], a["b"], a["tw"], a["rows"], a["d"], a["eps"], a["y"],
                                     a["ldy"], a["ty"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), sb.SDS_EINVAL), (dict(y=None), sb.SDS_EINVAL), (dict(ldx=63), sb.SDS_EINVAL),
    (dict(ldy=63), sb.SDS_EINVAL), (dict(rows=-1), sb.SDS_EINVAL), (dict(rows=(1 << 30) + 1), sb.SDS_EINVAL),
    (dict(d=0), sb.SDS_EINVAL), (dict(d=-3), sb.SDS_EINVAL), (dict(eps=-1e-6), sb.SDS_EINVAL),
    (dict(eps=float("nan")), sb.SDS_EINVAL), (dict(eps=float("inf")), sb.SDS_EINVAL),
    (dict(tx=3), sb.SDS_EUNSUPPORTED), (dict(ty=-1), sb.SDS_EUNSUPPORTED), (dict(tw=7), sb.SDS_EUNSUPPORTED),
    (dict(tx=sb.SDS_BF16, ty=sb.SDS_F32), sb.SDS_EUNSUPPORTED),     # only float rows change their type
    (dict(tx=sb.SDS_BF16, ty=sb.SDS_F16), sb.SDS_EUNSUPPORTED),
    (dict(x=X + 2), sb.SDS_EINVAL), (dict(y=Y + 1, ty=sb.SDS_BF16), sb.SDS_EINVAL), (dict(w=W + 2), sb.SDS_EINVAL),
    (dict(mean=M + 2), sb.SDS_EINVAL),
])
def test_layer_norm_refusals(kw, code):
    assert _norm(**kw) == code


def test_layer_norm_of_no_rows_does_nothing():
    assert _norm(rows=0, x=None, y=None, mean=None, rstd=None) == sb.SDS_OK


def _norm_bwd(**kw):
    a = dict(dy=Y, lddy=64, ty=sb.SDS_F32, x=X, ldx=64, tx=sb.SDS_F32, w=W, tw=sb.SDS_F32, mean=M, rstd=R, rows=4, d=64,
             dx=B, lddx=64, dw=0x200000, db=0x300000, ws=WS, bytes=1 << 30)
    a.update(kw)
    return sds.load().sds_layer_norm_backward(a["dy"], a["lddy"], a["ty"], a["x"], a["ldx"], a["tx"], a["w"], a["tw"],
                                              a["mean"], a["rstd"], a["rows"], a["d"], a["dx"], a["lddx"], a["dw"],
                                              a["db"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), sb.SDS_EINVAL), (dict(x=None), sb.SDS_EINVAL), (dict(lddy=10), sb.SDS_EINVAL),
    (dict(lddx=10), sb.SDS_EINVAL), (dict(mean=None), sb.SDS_EINVAL), (dict(rstd=None), sb.SDS_EINVAL),
    (dict(ws=None), sb.SDS_ENOMEM), (dict(ws=WS + 16), sb.SDS_ENOMEM), (dict(bytes=100), sb.SDS_ENOMEM),
    (dict(tx=sb.SDS_F16, ty=sb.SDS_F32), sb.SDS_EUNSUPPORTED), (dict(d=0), sb.SDS_EINVAL), (dict(rows=-1), sb.SDS_EINVAL),
    (dict(dw=0x200002), sb.SDS_EINVAL), (dict(dx=B + 2), sb.SDS_EINVAL),
])
def test_layer_norm_backward_refusals(kw, code):
    assert _norm_bwd(**kw) == code


def test_layer_norm_backward_without_a_wanted_gradient_does_nothing():
    assert _norm_bwd(dx=None, dw=None, db=None) == sb.SDS_OK


def test_layer_norm_workspace():
    n = C.c_size_t(0)
    f = sds.load().sds_layer_norm_workspace_bytes
    assert f(16, 64, None) == sb.SDS_EINVAL and f(-1, 64, C.byref(n)) == sb.SDS_EINVAL and f(1, 0, C.byref(n)) == sb.SDS_EINVAL
    for rows, d in ((0, 1), (1, 1), (5, 7), (1000, 64), (100000, 2048), (3, 16384), (7, 16385), (2, 100000)):
        assert f(rows, d, C.byref(n)) == sb.SDS_OK and n.value >= 2 * d * 4 and n.value % 256 == 0


def _ffn(**kw):
    a = dict(x=X, ldx=64, t=sb.SDS_BF16, rows=4, d=64, f=128, wg=W, wu=B, wd=M, act=0, y=Y, ldy=64, keep=None, ws=WS,
             bytes=1 << 30)
    a.update(kw)
    return sds.load().sds_gated_ffn(a["x"], a["ldx"], a["t"], a["rows"], a["d"], a["f"], a["wg"], a["wu"], a["wd"], a["act"],
                                    a["y"], a["ldy"], a["keep"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), sb.SDS_EINVAL), (dict(y=None), sb.SDS_EINVAL), (dict(wg=None), sb.SDS_EINVAL),
    (dict(wu=None), sb.SDS_EINVAL), (dict(wd=None), sb.SDS_EINVAL), (dict(rows=-1), sb.SDS_EINVAL),
    (dict(d=0), sb.SDS_EINVAL), (dict(f=-8), sb.SDS_EINVAL), (dict(ldx=56), sb.SDS_EINVAL), (dict(ldy=56), sb.SDS_EINVAL),
    (dict(d=60), sb.SDS_EUNSUPPORTED), (dict(f=100), sb.SDS_EUNSUPPORTED), (dict(ldx=68), sb.SDS_EUNSUPPORTED),
    (dict(ldy=68), sb.SDS_EUNSUPPORTED), (dict(x=X + 8), sb.SDS_EUNSUPPORTED), (dict(wd=M + 2), sb.SDS_EUNSUPPORTED),
    (dict(y=Y + 8), sb.SDS_EUNSUPPORTED), (dict(t=sb.SDS_F32), sb.SDS_EUNSUPPORTED), (dict(t=9), sb.SDS_EUNSUPPORTED),
    (dict(act=3), sb.SDS_EUNSUPPORTED), (dict(act=-1), sb.SDS_EUNSUPPORTED), (dict(ws=None), sb.SDS_ENOMEM),
    (dict(ws=WS + 128), sb.SDS_ENOMEM), (dict(bytes=255), sb.SDS_ENOMEM), (dict(keep=R + 16), sb.SDS_ENOMEM),
])
def test_gated_ffn_refusals(kw, code):
    assert _ffn(**kw) == code


def _ffn_bwd(**kw):
    a = dict(dy=Y, lddy=64, x=X, ldx=64, t=sb.SDS_BF16, rows=4, d=64, f=128, wg=W, wu=B, wd=M, keep=R, dx=0x200000, lddx=64,
             dwg=0x300000, dwu=0x400000, dwd=0x500000, ws=WS, bytes=1 << 30)
    a.update(kw)
    return sds.load().sds_gated_ffn_backward(a["dy"], a["lddy"], a["x"], a["ldx"], a["t"], a["rows"], a["d"], a["f"], a["wg"],
                                             a["wu"], a["wd"], a["keep"], a["dx"], a["lddx"], a["dwg"], a["dwu"],
                                             a["dwd"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), sb.SDS_EINVAL), (dict(x=None), sb.SDS_EINVAL), (dict(keep=None), sb.SDS_EINVAL),
    (dict(wd=None), sb.SDS_EINVAL), (dict(keep=R + 64), sb.SDS_ENOMEM), (dict(ws=None), sb.SDS_ENOMEM),
    (dict(bytes=1024), sb.SDS_ENOMEM), (dict(lddy=68), sb.SDS_EUNSUPPORTED), (dict(lddx=68), sb.SDS_EUNSUPPORTED),
    (dict(dwg=0x300008), sb.SDS_EUNSUPPORTED), (dict(t=sb.SDS_F32), sb.SDS_EUNSUPPORTED), (dict(d=12), sb.SDS_EUNSUPPORTED),
])
def test_gated_ffn_backward_refusals(kw, code):
    assert _ffn_bwd(**kw) == code


def test_gated_ffn_sizes():
    s = sds.gated_ffn_bytes(100, 64, 128)
    assert s.forward_bytes >= 100 * 128 * 2 and s.backward_bytes >= 2 * 100 * 128 * 2
    assert s.keep_bytes >= 100 * 128 * (2 + 8) and s.forward_keep_bytes <= s.forward_bytes
    assert sds.load().sds_gated_ffn_bytes(1, 64, 128, None) == sb.SDS_EINVAL
    for bad in ((-1, 64, 128), (1, 0, 8), (1, 8, -8)):
        with pytest.raises(sds.SdsError):
            sds.gated_ffn_bytes(*bad)
    with pytest.raises(sds.SdsError):
        sds.gated_ffn_bytes(1, 65, 128)
    big = sds.gated_ffn_bytes(1 << 20, 4096, 16384)               # sizes past 32 bits
    assert big.keep_bytes == (1 << 34) * 10 + 256
    assert sds.load().sds_gated_ffn_status(None, None) == sb.SDS_EINVAL


def test_host_checks_of_the_tensor_functions():
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        sds.layer_norm(x)                                           # not a CUDA tensor
    with pytest.raises(ValueError):
        sds.gated_ffn(x, x, x, x)
    for call in (lambda: sds.layer_norm(None), lambda: sds.layer_norm([1.0]), lambda: sds.gated_ffn(x, x, x, x, "relu"),
                 lambda: sds.layer_norm_backward(x, x, None, x, x), lambda: sds.gated_ffn_backward(x, x, x, x, x, x)):
        with pytest.raises(ValueError):
            call()


def _gated_den(d=64, f=128, act=0, nblock=2, drop=None, shift=0):
    n = 3 * nblock
    W = (C.c_void_p * n)(*[0x100000 + 0x1000 * i + shift for i in range(n)])
    if drop is not None:
        W[drop] = None
    norm = (C.c_void_p * (2 * nblock))(*([None] * (2 * nblock)))
    temb = (C.c_void_p * nblock)(*([None] * nblock))
    dims = (C.c_int32 * 3)(d, f, act)
    den = sb.SdsDenoiser()
    den.kind, den.nlayer = sb.SDS_DEN_GATED, nblock
    den.W_dev, den.bias_dev, den.temb_dev, den.dims = (C.cast(v, C.c_void_p) for v in (W, norm, temb, dims))
    return den, (W, norm, temb, dims)


def test_gated_denoiser_validation():
    import numpy as np
    a = np.full(5, 0.5, np.float32)
    sch = sb.SdsSchedule(5, a.ctypes.data, a.ctypes.data, a.ctypes.data, None, 0)
    n = C.c_size_t(0)
    ask = lambda den, d=64: sds.load().sds_workspace_bytes(C.byref(sch), C.byref(den[0]), 8, d, 4, C.byref(n))
    assert ask(_gated_den()) == sb.SDS_OK
    assert n.value >= 8 * 4 * (64 * 4 * 2 + 64 * 2 + 128 * 2)      # rows and outputs, normed and hidden rows
    assert ask(_gated_den(d=128)) == sb.SDS_EINVAL                  # another width than the context's
    assert ask(_gated_den(f=0)) == sb.SDS_EINVAL and ask(_gated_den(nblock=2, drop=4)) == sb.SDS_EINVAL
    assert ask(_gated_den(f=100)) == sb.SDS_EUNSUPPORTED and ask(_gated_den(act=7)) == sb.SDS_EUNSUPPORTED
    assert ask(_gated_den(d=60), 60) == sb.SDS_EUNSUPPORTED and ask(_gated_den(shift=8)) == sb.SDS_EUNSUPPORTED
    assert ask(_gated_den(d=16392), 16392) == sb.SDS_EUNSUPPORTED


def test_oracle_gated_block_by_hand():
    """One block on a row of two, worked out on paper: the norm of (1, 3) is (-1, 1) up to eps, gate and up pick its
    elements, and the product with Wd is added to the row."""
    import math
    from oracle import sds_oracle as o
    eye = [[1.0, 0.0], [0.0, 1.0]]
    got = o.gated_forward([0.5, 2.5], 1, [eye], [eye], [[[2.0, 0.0], [0.0, 1.0]]], [None], [None], [[[0.0, 0.0], [0.5, 0.5]]], "silu", eps=0.0)
    h = (1.0 / (1.0 + math.e)) , 1.0 / (1.0 + math.exp(-1.0))        # silu(-1) * -1, silu(1) * 1
    h = o.bf16_round(o.np.array(h))
    assert abs(got[0] - (1.0 + 2.0 * h[0])) < 1e-12 and abs(got[1] - (3.0 + h[1])) < 1e-12
    for name in ("silu", "gelu", "gelu_tanh"):
        assert o.gated_activation(o.np.zeros(3), name).tolist() == [0.0, 0.0, 0.0]
        assert abs(o.gated_activation(o.np.array([30.0]), name)[0] - 30.0) < 1e-9


def test_sizes_beyond_32_bit_counters_are_refused():
    big = (1 << 30) + 8
    n, s = C.c_size_t(0), sb.SdsGatedFfnSizes()
    assert _norm(d=big, ldx=big, ldy=big) == sb.SDS_EINVAL
    assert _norm_bwd(d=big, ldx=big, lddy=big, lddx=big, bytes=1 << 60) == sb.SDS_EINVAL
    assert sds.load().sds_layer_norm_workspace_bytes(1, big, C.byref(n)) == sb.SDS_EINVAL
    assert _ffn(d=big, ldx=big, ldy=big, bytes=1 << 60) == sb.SDS_EINVAL and _ffn(f=big, bytes=1 << 60) == sb.SDS_EINVAL
    assert _ffn_bwd(f=big, bytes=1 << 60) == sb.SDS_EINVAL
    assert sds.load().sds_gated_ffn_bytes(1, 64, big, C.byref(s)) == sb.SDS_EINVAL
