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
