"""Refusals and sizes of the linear layer, dropout and the residual norm, answered on the host before any launch (no GPU needed;
device pointers are numbers that nothing reads)."""
import ctypes as C
import math

import pytest

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb

X, W, B, T, S, R, Y, K, WS, D1, D2, D3 = (0x100000 + 0x10000 * i for i in range(12))
OK, INVAL, UNSUP, NOMEM = sb.SDS_OK, sb.SDS_EINVAL, sb.SDS_EUNSUPPORTED, sb.SDS_ENOMEM


def layer(a):
    return sb.SdsLinearLayer(a["k"], a["n"], a["steps"], a["t"], a["act"], a["w"], a["b"], a["bt"], a["table"])


LINEAR = dict(k=64, n=40, steps=5, t=sb.SDS_BF16, act=sb.SDS_ACT_SILU, w=W, b=B, bt=sb.SDS_F32, table=T, x=X, ldx=64, step=S, rows=4, res=R, ldr=40,
              y=Y, ldy=40, yt=sb.SDS_BF16, keep=K, ws=WS, bytes=1 << 30)


def _linear(**kw):
    a = dict(LINEAR, **kw)
    return sds.load().sds_linear(C.byref(layer(a)), a["x"], a["ldx"], a["step"], a["rows"], a["res"], a["ldr"], a["y"], a["ldy"], a["yt"],
                                 a["keep"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(w=None), INVAL), (dict(step=None), INVAL), (dict(rows=-1), INVAL), (dict(rows=(1 << 30) + 1), INVAL),
    (dict(k=0), INVAL), (dict(n=0), INVAL), (dict(steps=0), INVAL), (dict(steps=-1, table=None), INVAL), (dict(ldx=56), INVAL), (dict(ldy=39), INVAL),
    (dict(ldr=39), INVAL), (dict(y=Y + 1), INVAL), (dict(res=R + 1), INVAL), (dict(b=B + 2), INVAL), (dict(table=T + 1), INVAL), (dict(step=S + 2), INVAL),
    (dict(yt=sb.SDS_F32, y=Y + 2), INVAL), (dict(k=60), UNSUP), (dict(ldx=68), UNSUP), (dict(x=X + 8), UNSUP), (dict(w=W + 8), UNSUP), (dict(t=sb.SDS_F32), UNSUP),
    (dict(t=9), UNSUP), (dict(bt=9), UNSUP), (dict(yt=sb.SDS_F16), UNSUP), (dict(yt=7), UNSUP), (dict(act=4), UNSUP), (dict(act=-1), UNSUP),
    (dict(steps=65536), UNSUP), (dict(ws=None), NOMEM), (dict(ws=WS + 128), NOMEM), (dict(bytes=255), NOMEM), (dict(keep=K + 16), NOMEM),
])
def test_linear_refusals(kw, code):
    assert _linear(**kw) == code


def _linear_bwd(**kw):
    a = dict(LINEAR, dx=D1, lddx=64, dw=D2, db=D3, dt=D3 + 0x10000, dy=Y, lddy=40)
    a.update(kw)
    return sds.load().sds_linear_backward(C.byref(layer(a)), a["dy"], a["lddy"], a["yt"], a["x"], a["ldx"], a["step"], a["rows"], a["keep"], a["dx"],
                                          a["lddx"], a["dw"], a["db"], a["dt"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), INVAL), (dict(x=None), INVAL), (dict(keep=None), INVAL), (dict(w=None), INVAL), (dict(step=None), INVAL), (dict(lddy=39), INVAL),
    (dict(lddx=56), INVAL), (dict(b=None), INVAL), (dict(table=None, steps=0), INVAL), (dict(db=D3 + 2), INVAL), (dict(dt=D3 + 1), INVAL), (dict(dy=Y + 1), INVAL),
    (dict(lddx=68), UNSUP), (dict(dx=D1 + 8), UNSUP), (dict(dw=D2 + 8), UNSUP), (dict(yt=sb.SDS_F16), UNSUP), (dict(t=sb.SDS_F32), UNSUP),
    (dict(keep=K + 64), NOMEM), (dict(ws=None), NOMEM), (dict(bytes=512), NOMEM),
])
def test_linear_backward_refusals(kw, code):
    assert _linear_bwd(**kw) == code


def test_linear_sizes():
    f, s = sds.load().sds_linear_bytes, sb.SdsLinearSizes()
    a = layer(LINEAR)
    assert f(C.byref(a), 100, None) == INVAL and f(None, 100, C.byref(s)) == INVAL and f(C.byref(a), -1, C.byref(s)) == INVAL
    for rows in (0, 1, 7, 100, 100000):
        for n in (1, 40, 41, 5000):
            a = layer(dict(LINEAR, n=n))
            assert f(C.byref(a), rows, C.byref(s)) == OK
            assert s.keep_bytes >= rows * n * 4 and s.backward_bytes >= rows * n * 2 + rows * 4 and s.forward_bytes >= 4
            assert not any(v % 256 for v in (s.keep_bytes, s.forward_bytes, s.backward_bytes))
    a = layer(dict(LINEAR, act=sb.SDS_ACT_NONE))
    assert f(C.byref(a), 100, C.byref(s)) == OK and s.keep_bytes == 0
    a = layer(dict(LINEAR, n=1 << 20, table=None))
    assert f(C.byref(a), 1 << 20, C.byref(s)) == OK and s.keep_bytes == 1 << 42          # sizes past 32 bits
    assert sds.load().sds_linear_status(None, None) == INVAL


def spec(**kw):
    a = dict(p=0.1, seed=1, step=2, step_dev=None, row0=0)
    a.update(kw)
    return sb.SdsDropoutSpec(a["p"], a["seed"], a["step"], a["step_dev"], a["row0"])


def _dropout(sp=None, **kw):
    a = dict(x=X, ldx=40, tx=sb.SDS_BF16, rows=4, d=40, res=R, ldr=40, y=Y, ldy=40, ty=sb.SDS_F32)
    a.update(kw)
    sp = spec() if sp is None else sp
    return sds.load().sds_dropout(C.byref(sp), a["x"], a["ldx"], a["tx"], a["rows"], a["d"], a["res"], a["ldr"], a["y"], a["ldy"], a["ty"], None)


BAD_SPECS = [dict(p=-0.1), dict(p=1.5), dict(p=math.nan), dict(p=math.inf), dict(step=-1), dict(row0=-1), dict(row0=1 << 56), dict(row0=(1 << 56) - 3), dict(step_dev=S + 2)]


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(rows=-1), INVAL), (dict(d=0), INVAL), (dict(ldx=39), INVAL), (dict(ldy=39), INVAL), (dict(ldr=39), INVAL),
    (dict(x=X + 1), INVAL), (dict(y=Y + 2), INVAL), (dict(rows=(1 << 30) + 1), INVAL), (dict(tx=9), UNSUP), (dict(ty=9), UNSUP), (dict(ty=sb.SDS_F16), UNSUP),
])
def test_dropout_refusals(kw, code):
    assert _dropout(**kw) == code


@pytest.mark.parametrize("kw", BAD_SPECS, ids=str)
def test_dropout_refuses_bad_draws(kw):
    assert _dropout(spec(**kw)) == INVAL
    assert _norm(drop=spec(**kw)) == INVAL
    assert sds.load().sds_dropout(None, X, 40, 0, 4, 40, None, 0, Y, 40, 0, None) == INVAL


NORM = dict(rows=12, groups=3, d=40, rt=sb.SDS_F32, ht=sb.SDS_BF16, kind=0, post=1, alpha=1.0, eps=1e-5, w=W, b=B, pw=T, wt=sb.SDS_F32, gate=D1, scale=D2,
            shift=D3, ldg=40, lds=120, ldh_=40, ct=sb.SDS_BF16, drop=None, r=X, ldr=40, h=R, ldh=40, out=Y, ldo=40, n=S, ldn=40, keep=K, ws=WS, bytes=1 << 30)


def norm_op(a):
    return sb.SdsResidualNormOp(a["rows"], a["groups"], a["d"], a["rt"], a["ht"], a["kind"], a["post"], a["alpha"], a["eps"], a["w"], a["b"], a["pw"], a["wt"],
                                a["gate"], a["scale"], a["shift"], a["ldg"], a["lds"], a["ldh_"], a["ct"], a["drop"] or spec(p=0.0))


def _norm(**kw):
    a = dict(NORM, **kw)
    return sds.load().sds_residual_norm(C.byref(norm_op(a)), a["r"], a["ldr"], a["h"], a["ldh"], a["out"], a["ldo"], a["n"], a["ldn"], a["keep"], None)


COMMON = [
    (dict(r=None), INVAL), (dict(rows=-1), INVAL), (dict(rows=13), INVAL), (dict(groups=0), INVAL), (dict(d=0), INVAL), (dict(ldr=39), INVAL), (dict(ldh=39), INVAL),
    (dict(kind=2), INVAL), (dict(eps=-1.0), INVAL), (dict(eps=math.nan), INVAL), (dict(alpha=math.inf), INVAL), (dict(w=W + 2), INVAL), (dict(gate=D1 + 1), INVAL),
    (dict(ldg=39), INVAL), (dict(lds=39), INVAL), (dict(ldh_=39), INVAL), (dict(d=16392, ldr=16392, ldh=16392), UNSUP), (dict(rt=sb.SDS_BF16, ht=sb.SDS_F32), UNSUP),
    (dict(rt=9), UNSUP), (dict(wt=9), UNSUP), (dict(ct=9), UNSUP), (dict(ldr=1 << 31), UNSUP), (dict(ldg=1 << 31), UNSUP), (dict(keep=K + 16), NOMEM),
]


@pytest.mark.parametrize("kw,code", COMMON + [(dict(n=None), INVAL), (dict(out=None), INVAL), (dict(ldo=39), INVAL), (dict(ldn=39), INVAL), (dict(n=S + 1), INVAL)])
def test_residual_norm_refusals(kw, code):
    assert _norm(**kw) == code


def _norm_bwd(**kw):
    a = dict(NORM, dn=S, lddn=40, dout=Y, lddout=40, g={})
    a.update(kw)
    g = dict(dr_dev=0x900000, ld_dr=40, dh_dev=0x910000, ld_dh=40, dw_dev=0x920000, db_dev=0x930000, dpost_w_dev=0x940000, dgate_dev=0x950000,
             dscale_dev=0x960000, dshift_dev=0x970000, ld_dgate=40, ld_dscale=40, ld_dshift=40)
    g.update(a["g"])
    return sds.load().sds_residual_norm_backward(C.byref(norm_op(a)), a["dn"], a["lddn"], a["dout"], a["lddout"], a["r"], a["ldr"], a["h"], a["ldh"], a["keep"],
                                                 C.byref(sb.SdsResidualNormGrads(**g)), a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(dn=None), INVAL), (dict(lddn=39), INVAL), (dict(lddout=39), INVAL), (dict(h=None), INVAL), (dict(post=0), INVAL), (dict(keep=None), INVAL),
    (dict(g=dict(ld_dr=39)), INVAL), (dict(g=dict(dh_dev=0x910001)), INVAL), (dict(g=dict(dw_dev=0x920002)), INVAL), (dict(g=dict(ld_dgate=39)), INVAL),
    (dict(g=dict(dshift_dev=0x970001)), INVAL), (dict(ws=None), NOMEM), (dict(ws=WS + 64), NOMEM), (dict(bytes=256), NOMEM),
])
def test_residual_norm_backward_refusals(kw, code):
    assert _norm_bwd(**kw) == code


def test_residual_norm_backward_without_a_wanted_gradient_does_nothing():
    none = {k: None for k in ("dr_dev", "dh_dev", "dw_dev", "db_dev", "dpost_w_dev", "dgate_dev", "dscale_dev", "dshift_dev")}
    assert _norm_bwd(g=none) == OK


def test_residual_norm_sizes():
    f, s = sds.load().sds_residual_norm_bytes, sb.SdsResidualNormSizes()
    assert f(C.byref(norm_op(NORM)), None) == INVAL and f(None, C.byref(s)) == INVAL
    for rows, groups, d in ((0, 3, 40), (12, 12, 40), (12, 1, 7), (100000, 10, 64), (2048, 64, 16384)):
        assert f(C.byref(norm_op(dict(NORM, rows=rows, groups=groups, d=d, ldg=d, lds=d, ldh_=d))), C.byref(s)) == OK
        assert s.keep_bytes == rows * 32 and s.backward_bytes >= (3 * d * 4 if rows else 1) and s.backward_bytes % 256 == 0


def test_host_checks_of_the_tensor_functions():
    import torch
    x, w = torch.zeros(4, 64), torch.zeros(8, 64)
    bad = [lambda: sds.linear(x, w), lambda: sds.linear(None, w), lambda: sds.linear(x, w, activation="tanh"), lambda: sds.linear_backward(x, x, w, x),
           lambda: sds.dropout(x, 0.1, 1), lambda: sds.dropout([1.0], 0.1, 1), lambda: sds.dropout_backward(x, 0.1, 1), lambda: sds.residual_norm(x, x),
           lambda: sds.residual_norm(x, kind="group"), lambda: sds.residual_norm_backward(x, x, x, x, x), lambda: sds.residual_norm(None)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
