"""Residual norm and dropout on the GPU against their definitions in 64 bits.

Tolerances, derived from the arithmetic. u = 2^-24. A row's sums: eight terms in a thread, five steps in a warp, at most 64 warps'
sums: (8 + 5 + 64) u, S below, of the sum of the terms' sizes. Errors of a row's values reach its norm through the mean and the size, of which
the bounds below take the first order. Sums over rows: at most `rows` terms one after the other. Every output is rounded once
to its type (half a step).
"""
import numpy as np
import pytest
import torch

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
S = 80 * U
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).tiny * torch.finfo(t).eps      # the step of the subnormal range


def close(got, want, bound, what=""):
    """got within half a step of its type of want, and `bound` of error before that rounding."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g = got.double()
    assert torch.isfinite(g).all(), what
    over = (g - want).abs() / ((want.abs() + bound) * half(got.dtype) + bound + tiny(got.dtype))
    assert over.max() <= 1.0, (what, float(over.max()), int(over.argmax()))


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def factor(rows, d, p, seed, step, row0=0):
    """D in 64 bits, from the generator's definition, counter by counter on the host."""
    thr = round(p * 65536)
    if thr == 65536:
        return torch.zeros(rows, d, dtype=torch.float64, device="cuda")
    nb = (d + 7) // 8
    row = np.repeat(np.arange(row0, row0 + rows, dtype=np.uint64), nb)
    c = [np.tile(np.arange(nb, dtype=np.uint64), rows), np.full(rows * nb, step, np.uint64), row & np.uint64(0xFFFFFFFF),
         np.uint64(3) + np.uint64(256) * (row >> np.uint64(32))]
    k0, k1, m = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    draws = np.stack([w for v in c for w in (v & np.uint64(0xFFFF), v >> np.uint64(16))], axis=1).reshape(rows, nb * 8)[:, :d]
    return torch.from_numpy((draws >= thr).astype(np.float64) * (65536.0 / (65536 - thr))).cuda()


# ---------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------

DROP_TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16), (BF16, F32), (F16, F32)]


@pytest.mark.parametrize("tx,ty", DROP_TYPES)
@pytest.mark.parametrize("rows,d,p", [(1, 1, 0.5), (3, 7, 0.1), (64, 2048, 0.1), (1021, 1001, 0.3), (33, 64, 0.0), (5, 40, 1.0), (700, 256, 0.999), (2, 100003, 0.25)])
def test_dropout(rows, d, p, tx, ty):
    r = gen(rows + d)
    x = r(rows, d).to(tx)
    seed, step = 0x123456789ABCDEF0 + d, 5
    D = factor(rows, d, p, seed, step)
    want = D * x.double()
    if tx == ty:
        y = sds.dropout(x, p, seed, step)
        close(y, want, U * want.abs())
        assert torch.equal(sds.dropout_backward(x, p, seed, step), y)
        assert ((y == 0) == ((D == 0) | (x == 0))).all()
    else:
        close(sds.dropout_backward(x, p, seed, step, out_dtype=ty), want, U * want.abs())
    if tx == ty or ty == F32:
        res = r(rows, d).to(ty)
        y = sds.dropout(x, p, seed, step, residual=res)
        assert y.dtype == ty
        close(y, want + res.double(), U * (want.abs() + (want + res.double()).abs()))


def test_dropout_draws():
    """Another step, seed or row draws another mask; shards draw what the whole draws; the mean is kept."""
    x = torch.ones(512, 4096, device="cuda")
    y = sds.dropout(x, 0.2, 7, 3)
    thr = round(0.2 * 65536)
    assert abs(float((y == 0).double().mean()) - thr / 65536) < 5 * (0.2 * 0.8 / y.numel()) ** 0.5
    assert abs(float(y.double().mean()) - 1) < 5 * (0.25 / y.numel()) ** 0.5
    for other in (sds.dropout(x, 0.2, 8, 3), sds.dropout(x, 0.2, 7 + (1 << 40), 3), sds.dropout(x, 0.2, 7, 4), sds.dropout(x, 0.2, 7, 3, row0=1)):
        assert abs(float(((other == 0) & (y == 0)).double().mean()) - (thr / 65536) ** 2) < 1e-3
    parts = torch.cat([sds.dropout(x[:100], 0.2, 7, 3), sds.dropout(x[100:], 0.2, 7, 3, row0=100)])
    assert torch.equal(parts, y)
    far = (1 << 45) + 12345
    close(sds.dropout(x[:3], 0.2, 7, 3, row0=far), factor(3, 4096, 0.2, 7, 3, far), torch.zeros(3, 4096, device="cuda", dtype=torch.float64) + U * 2)
    # a row's mask does not depend on its length, nor on where its rows lie
    assert torch.equal(sds.dropout(x[:, :1001], 0.2, 7, 3), y[:, :1001])


def test_dropout_step_of_a_captured_graph():
    x = gen(1)(40, 200)
    step = torch.zeros(1, device="cuda", dtype=torch.int32)
    y = sds.dropout(x, 0.3, 9, step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sds.dropout(x, 0.3, 9, step)
        dx = sds.dropout_backward(x, 0.3, 9, step)
    for k in (0, 1, 77):
        step.fill_(k)
        graph.replay()
        assert torch.equal(y, sds.dropout(x, 0.3, 9, k)) and torch.equal(dx, y)


def test_dropout_in_place_strided_and_special():
    r = gen(2)
    big = r(50, 130).to(BF16)
    x = big[:, 1:101]
    want = sds.dropout(x.contiguous(), 0.4, 3)
    out = torch.full((50, 120), 7.0, device="cuda", dtype=BF16)
    sds.dropout(x, 0.4, 3, out=out[:, 4:104])
    assert torch.equal(out[:, 4:104], want) and (out[:, :4] == 7).all() and (out[:, 104:] == 7).all()
    rest = big[:, 101:].clone()
    sds.dropout(x, 0.4, 3, out=x)
    assert torch.equal(x, want) and torch.equal(big[:, 101:], rest)
    res = r(50, 96)
    want = sds.dropout(r(50, 96), 0.4, 3, residual=res)
    x = gen(2)
    for d in (96, 97):                                   # inf and NaN behind the mask are gone, others stay
        x = torch.full((40, d), float("nan"), device="cuda")
        y = sds.dropout(x, 0.5, 4, residual=torch.ones(40, d, device="cuda"))
        D = factor(40, d, 0.5, 4, 0)
        assert (y[D == 0] == 1).all() and torch.isnan(y[D != 0]).all()
    assert sds.dropout(torch.empty(0, 8, device="cuda"), 0.5, 1).shape == (0, 8)
    assert sds.dropout(torch.ones(3, 4, 5, device="cuda"), 0.5, 1).shape == (3, 4, 5)


def test_dropout_refusals():
    x = torch.ones(4, 8, device="cuda")
    for call in (lambda: sds.dropout(x, -0.1, 1), lambda: sds.dropout(x, 1.1, 1), lambda: sds.dropout(x, float("nan"), 1), lambda: sds.dropout(x, 0.1, -1),
                 lambda: sds.dropout(x, 0.1, 1 << 64), lambda: sds.dropout(x, 0.1, 1, -1), lambda: sds.dropout(x, 0.1, 1, 1 << 31), lambda: sds.dropout(x, 0.1, 1, row0=-1),
                 lambda: sds.dropout(x, 0.1, 1, torch.zeros(1, device="cuda")), lambda: sds.dropout(x, 0.1, 1, torch.zeros(2, device="cuda", dtype=torch.int32)),
                 lambda: sds.dropout(x, 0.1, 1, torch.zeros(1, dtype=torch.int32)), lambda: sds.dropout(x.cpu(), 0.1, 1), lambda: sds.dropout(x.double(), 0.1, 1),
                 lambda: sds.dropout(x, 0.1, 1, residual=x[:2]), lambda: sds.dropout(x, 0.1, 1, out=x[:2]), lambda: sds.dropout(x[:, ::2], 0.1, 1),
                 lambda: sds.dropout(x[:1].expand(4, 8), 0.1, 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sds.SdsError) as e:
        sds.dropout(x.bfloat16(), 0.1, 1, residual=x.half())
    assert e.value.code == sb.SDS_EUNSUPPORTED
    with pytest.raises(sds.SdsError) as e:
        sds.dropout(x, 0.1, 1, row0=1 << 56)
    assert e.value.code == sb.SDS_EINVAL


# ---------------------------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------------------------


def xhat64(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


class Norms64:
    """The operator in 64 bits with autograd, and bounds of every output's error before its last rounding."""

    def __init__(self, s, eps=1e-5):
        self.s, kind = s, s["kind"]
        rows, d = s["r"].shape
        self.rows, self.d, self.per = rows, d, rows // s["groups"]
        names = [n for n in ("r", "h", "weight", "bias", "scale", "shift", "gate", "post_weight") if s[n] is not None]
        self.v = {n: s[n].double().requires_grad_(True) for n in names}
        v, spread = self.v, lambda t: t.repeat_interleave(self.per, 0)  # noqa: E731
        mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
        size = lambda t, c: 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)  # noqa: E731
        centred = lambda t: t - mean(t) if kind == "layer" else t  # noqa: E731
        self.out = v["r"]
        self.eout = torch.zeros(rows, d, device="cuda", dtype=torch.float64)
        if s["h"] is not None:
            self.D = factor(rows, d, s["p"], s["seed"], s["step"], s["row0"]) if s["p"] else torch.ones(rows, d, device="cuda", dtype=torch.float64)
            self.gate = spread(v["gate"]) if "gate" in v else torch.ones(1, device="cuda", dtype=torch.float64)
            self.wp = v["post_weight"] if "post_weight" in v else torch.ones(d, device="cuda", dtype=torch.float64)
            if s["post"]:
                self.phat = xhat64(v["h"], kind, eps)
                self.ps = size(v["h"], centred(v["h"])).detach()
                self.eph = S * (self.phat.abs() + 1)
                q, eq = self.phat * self.wp, self.eph * self.wp.abs()
            else:
                self.phat, self.eph = v["h"], torch.zeros_like(v["h"])
                q, eq = v["h"], 0.0
            self.k = s["alpha"] * self.gate * self.D
            self.out = v["r"] + self.k * q
            # (alpha itself is a float)
            self.eout = self.k.abs() * eq + 5 * U * (self.k * q).abs() + U * self.out.abs()
        self.xhat = xhat64(self.out, kind, eps)
        self.rs = size(self.out, centred(self.out)).detach()
        xa = self.xhat.detach().abs()
        ev = self.eout.detach()
        self.exh = S * (xa + 1) + self.rs * (ev + mean(ev) + xa * mean(xa * ev))
        self.ers = 2 * S + self.rs * mean(xa * ev)
        w = v["weight"] if "weight" in v else torch.ones(d, device="cuda", dtype=torch.float64)
        b = v["bias"] if "bias" in v else torch.zeros(d, device="cuda", dtype=torch.float64)
        self.f = 1 + spread(v["scale"]) if "scale" in v else torch.ones(1, device="cuda", dtype=torch.float64)
        sh = spread(v["shift"]) if "shift" in v else torch.zeros(1, device="cuda", dtype=torch.float64)
        self.w, self.b = w, b
        u = self.xhat * w + b
        self.eu = self.exh * w.abs() + 2 * U * (xa * w.abs() + b.abs())
        self.n = u * self.f + sh
        self.en = self.eu * self.f.abs() + 3 * U * ((u * self.f).abs() + sh.abs())
        self.u = u

    def backward(self, dn, dr):
        s, v = self.s, self.v
        heads, seeds = [self.n], [dn.double()]
        if dr is not None:
            heads, seeds = heads + [self.out], seeds + [dr.double()]
        if s["h"] is None and dr is not None:
            heads[1] = v["r"] * 1.0
        grads = dict(zip(v, torch.autograd.grad(heads, list(v.values()), seeds)))
        with torch.no_grad():
            mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
            groups = lambda t: t.reshape(s["groups"], self.per, self.d).sum(1)  # noqa: E731
            sr = (self.rows + 100) * U
            xa, da = self.xhat.abs(), dn.double().abs()
            dx = da * (self.f * self.w).abs()
            c1, c2 = mean(dx), mean(dx * xa)
            edx = 4 * U * dx
            ec2 = S * c2 + mean(dx * self.exh) + mean(edx * xa)
            body = dx + c1 + xa * c2
            eg = self.rs * (edx + S * c1 + mean(edx) + self.exh * c2 + xa * ec2 + 4 * U * body) + self.ers * self.rs * body
            g = grads["r"].abs()
            eg = eg + U * (g + (0 if dr is None else dr.double().abs()))
            bounds = {"r": eg}
            eA, A = da * self.exh + 2 * U * da * xa, da * xa
            bounds["shift"] = groups(sr * da)
            bounds["scale"] = groups(da * self.eu + (sr + 4 * U) * da * (xa * self.w.abs() + self.b.abs()))
            bounds["weight"] = (self.f.abs() * (eA + (sr + 4 * U) * A)).sum(0)
            bounds["bias"] = (self.f.abs() * (sr + 2 * U) * da).sum(0)
            if s["h"] is not None:
                pa = self.phat.abs()
                gabs = self.rs * body + (0 if dr is None else dr.double().abs())
                C = gabs * self.D * pa
                eC = self.D * (eg * pa + gabs * self.eph) + (sr + 4 * U) * C
                bounds["gate"] = groups(abs(s["alpha"]) * self.wp.abs() * (eC + 4 * U * C))
                bounds["post_weight"] = (abs(s["alpha"]) * self.gate.abs() * (eC + 4 * U * C)).sum(0)
                dq, edq = self.k.abs() * gabs, self.k.abs() * (eg + 5 * U * gabs)
                if s["post"]:
                    dp, edp = dq * self.wp.abs(), edq * self.wp.abs() + U * dq * self.wp.abs()
                    c1, c2 = mean(dp), mean(dp * pa)
                    body = dp + c1 + pa * c2
                    ec2 = S * c2 + mean(dp * self.eph) + mean(edp * pa)
                    edq = self.ps * (edp + S * c1 + mean(edp) + self.eph * c2 + pa * ec2 + 4 * U * body) + 2 * S * self.ps * body
                bounds["h"] = edq
        return grads, bounds


ORDER = ("r", "h", "weight", "bias", "scale", "shift", "gate", "post_weight")


def make(rows, d, tr, th, seed, groups=1, kind="layer", h=True, weight=None, bias=None, mod=None, gate=None, post=False, post_weight=None, p=0.0, alpha=0.75):
    """Tensors of the call; weight, bias, mod, gate, post_weight: a type, or None."""
    r = gen(seed)
    s = dict(kind=kind, groups=groups, post=post, p=p, alpha=alpha, seed=seed, step=3, row0=0)
    s["r"] = (r(rows, d) * torch.exp(0.5 * r(rows, 1)) + r(rows, 1)).to(tr)
    s["h"] = r(rows, d).to(th) if h else None
    s["weight"] = (1 + 0.3 * r(d)).to(weight) if weight else None
    s["bias"] = (0.3 * r(d)).to(bias) if bias else None
    cond = 0.5 * r(groups, 3 * d)
    s["scale"], s["shift"] = (cond[:, :d].to(mod), cond[:, d:2 * d].to(mod)) if mod else (None, None)
    s["gate"] = cond[:, 2 * d:].to(gate) if gate else None
    s["post_weight"] = (1 + 0.3 * r(d)).to(post_weight) if post_weight else None
    s["dn"], s["dr"] = r(rows, d).to(th), r(rows, d).to(tr)
    return s


def keywords(s):
    return {k: s[k] for k in ("weight", "bias", "scale", "shift", "gate", "post", "post_weight", "kind", "alpha", "p", "seed", "step", "row0")}


def check(s, dr=True):
    th = s["dn"].dtype
    kw = keywords(s)
    od = {} if s["h"] is not None else {"out_dtype": th}
    ref = Norms64(s)
    out, n = sds.residual_norm(s["r"], s["h"], **kw, **od)
    assert n.dtype == th and out.dtype == s["r"].dtype
    close(out, ref.out.detach(), ref.eout.detach(), "out")
    close(n, ref.n.detach(), ref.en.detach(), "n")
    out2, n2, kept = sds.residual_norm(s["r"], s["h"], keep=True, **kw, **od)
    assert torch.equal(out, out2) and torch.equal(n, n2)
    got = sds.residual_norm_backward(s["dn"], s["dr"] if dr else None, s["r"], s["h"], kept, **kw)
    grads, bounds = ref.backward(s["dn"], s["dr"] if dr else None)
    for name, v in zip(ORDER, got):
        if s[name] is None:
            assert v is None, name
            continue
        assert v.dtype == s[name].dtype, name
        close(v, grads[name], bounds[name].detach(), name)
        off = float((v.double() - grads[name]).norm() / (grads[name].norm() + 1e-30))
        assert off <= 2 * half(v.dtype) + 3e-6 or v.numel() < 64, (name, off)
    return (out, n) + got


# every thread group at its edges, aligned and not
SIZES = [(1, 1), (3, 5), (70, 64), (33, 65), (19, 72), (6, 256), (300, 257), (9, 512), (12, 513), (9, 1000), (301, 1001), (6, 1024), (17, 2048), (8, 2049),
         (4, 4096), (3, 5000), (6, 8192), (4, 8193), (6, 16384), (3, 16383)]


@pytest.mark.parametrize("tr,th", TYPES)
@pytest.mark.parametrize("rows,d", SIZES)
def test_sizes(rows, d, tr, th):
    for kind in ("layer", "rms"):
        which = rows + d + (kind == "rms")
        groups = [1, rows, rows // 3 if rows % 3 == 0 else 1][which % 3]
        check(make(rows, d, tr, th, which, groups=groups, kind=kind, weight=F32, bias=F32, mod=th, gate=th, post=which % 2 == 0,
                   post_weight=F32 if which % 2 == 0 else None, p=0.2 if which % 4 < 2 else 0.0))


PARTS = [dict(), dict(weight=F32), dict(bias=BF16), dict(weight=F16, bias=F16), dict(mod=F32), dict(gate=BF16), dict(mod=F16, gate=F16), dict(post=True),
         dict(post=True, post_weight=BF16, weight=BF16), dict(p=0.3), dict(post=True, p=0.3, gate=F32, mod=F32, weight=F32, bias=F32),
         dict(h=False), dict(h=False, weight=F32, bias=F32), dict(h=False, mod=BF16)]


@pytest.mark.parametrize("part", PARTS, ids=str)
@pytest.mark.parametrize("rows,d,groups", [(48, 520, 1), (48, 520, 48), (48, 520, 6), (48, 333, 1), (48, 333, 48), (48, 333, 6)])
def test_every_part_alone_and_together(rows, d, groups, part):
    for kind in ("layer", "rms"):
        s = make(rows, d, F32, BF16, d, groups=groups, kind=kind, **part)
        check(s)
        check(s, dr=False)


@pytest.mark.parametrize("rows,d,groups", [(5000, 64, 1), (5000, 64, 5000), (5000, 64, 5), (5000, 64, 1250), (3000, 72, 2), (2400, 1001, 3), (2400, 1001, 800),
                                           (1200, 2048, 1), (1200, 2048, 4), (1200, 2048, 600), (640, 4096, 2), (400, 8192, 1), (300, 16384, 3), (300, 8200, 300),
                                           (4097, 40, 17), (10000, 8, 1), (60000, 16, 20000), (60000, 16, 15),
                                           (6000, 300, 2000)])
def test_sums_over_many_rows(rows, d, groups):
    """Workers with several rows, pieces of groups, whole groups per worker, rows that are groups; the same bits again."""
    s = make(rows, d, F32, BF16, rows + d, groups=groups, weight=F32, bias=F32, mod=BF16, gate=BF16, post=True, post_weight=F32, p=0.1)
    first = check(s)
    again = check(s)
    assert all(torch.equal(a, b) for a, b in zip(first, again) if a is not None)


def test_rows_far_from_zero():
    r = gen(4)
    for d in (64, 1001, 2048, 8192):
        x = (r(20, d) + 10000.0).contiguous()
        h = r(20, d)
        _, n, kept = sds.residual_norm(x, h, keep=True)
        want = xhat64(x.double() + h.double(), "layer", 1e-5)
        # the sum r + h is rounded at 1e4: 2^-11 of a row's spread; the norm adds its own few units
        assert float((n.double() - want).abs().max()) <= 1.05 * 10010 * U * 2 + S * 8
        n = sds.residual_norm(x)[1]
        assert float((n.double() - xhat64(x.double(), "layer", 1e-5)).abs().max()) <= S * 8


@pytest.mark.parametrize("d", [7, 64, 1024, 16384])
def test_special_rows(d):
    """Constant rows, zeros, infinities and NaN stay in their rows."""
    r = gen(5)
    x, h = r(12, d), r(12, d)
    want = sds.residual_norm(x, h, kind="rms")
    x[1] = 3.0
    h[1] = 0.0
    x[2], h[2] = 0.0, 0.0
    x[5, 0] = float("inf")
    h[7, d - 1] = float("nan")
    for kind in ("layer", "rms"):
        out, n = sds.residual_norm(x, h, kind=kind)
        assert torch.isfinite(n[[0, 1, 2, 3, 4, 6, 8, 9, 10, 11]]).all()
        assert (n[2] == 0).all() and not torch.isfinite(n[5]).all() and torch.isnan(n[7]).all()
        if kind == "layer":
            assert (n[1] == 0).all()
        else:
            rest = [0, 3, 4, 6, 8, 9, 10, 11]
            assert torch.equal(n[rest], want[1][rest])


@pytest.mark.parametrize("d,pad", [(64, 8), (1000, 3), (2048, 16), (16384, 8)])
def test_strided_rows_leave_the_rest(d, pad):
    r = gen(6)
    rows = 24
    x, h = r(rows, d + pad)[:, pad // 2:pad // 2 + d], r(rows, d + pad).to(BF16)[:, :d]
    cond = r(4, 3 * d + 5).to(BF16)
    kw = dict(gate=cond[:, :d], scale=cond[:, d:2 * d], shift=cond[:, 2 * d:3 * d])
    want = sds.residual_norm(x.contiguous(), h.contiguous(), **{k: v.contiguous() for k, v in kw.items()}, keep=True)
    stream, out = torch.full((rows, d + 7), 7.0, device="cuda"), torch.full((rows, d + 5), 7.0, device="cuda", dtype=BF16)
    got = sds.residual_norm(x, h, **kw, keep=True, stream_out=stream[:, 3:3 + d], out=out[:, 2:2 + d])
    assert torch.equal(got[0], want[0])
    # Rows that lie otherwise are dealt to the threads otherwise, and sums in another order need not be the same bits: each xhat is within
    # S (|xhat| + 1) of the exact one, so two of them are within twice that (|1 + scale| < 8, |shift| < 8 here); each is then rounded
    # to bf16 by at most half a step of itself.
    n, m = got[1].double(), want[1].double()
    assert ((n - m).abs() <= half(BF16) * (n.abs() + m.abs()) + 2 * S * 8 * (m.abs() + 16)).all()
    assert (stream[:, :3] == 7).all() and (stream[:, 3 + d:] == 7).all() and (out[:, :2] == 7).all() and (out[:, 2 + d:] == 7).all()
    dn, dr = r(rows, d + 1).to(BF16)[:, 1:], r(rows, d + 3)[:, :d]
    a = sds.residual_norm_backward(dn, dr, x, h, got[2], **kw)
    b = sds.residual_norm_backward(dn.contiguous(), dr.contiguous(), x.contiguous(), h.contiguous(), want[2], **kw)
    for p, q in zip(a, b):
        # (another way to deal columns to threads: the sums' order differs)
        assert (p is None) == (q is None) and (p is None or float((p.double() - q.double()).norm()) <= (half(p.dtype) * 2 + 1e-6) * float(q.double().norm()))


def test_outputs_in_the_place_of_inputs():
    for d in (520, 333):
        s = make(50, d, F32, BF16, 1, gate=BF16, mod=BF16)
        want = sds.residual_norm(s["r"], s["h"], **keywords(s))
        got = sds.residual_norm(s["r"], s["h"], **keywords(s), stream_out=s["r"], out=s["h"])
        assert got[0].data_ptr() == s["r"].data_ptr() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_dropout_inside_is_the_dropout_operator():
    for d in (256, 1001, 4096, 16384):
        r = gen(d)
        x, h = r(30, d), r(30, d)
        out, _ = sds.residual_norm(x, h, p=0.25, seed=99, step=4, row0=1 << 33)
        assert torch.equal(out, sds.dropout(h, 0.25, 99, 4, residual=x, row0=1 << 33))


def test_wanted_gradients():
    for groups, d in ((1, 264), (40, 264), (5, 264), (5, 99)):
        s = make(40, d, F32, BF16, 8, groups=groups, weight=F32, bias=F32, mod=BF16, gate=BF16, post=True, post_weight=F32, p=0.1)
        kw = keywords(s)
        kept = sds.residual_norm(s["r"], s["h"], keep=True, **kw)[2]
        every = sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, **kw)
        for i in range(8):
            one = sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, want=[k == i for k in range(8)], **kw)
            for k in range(8):
                assert one[k] is None if k != i else one[k].shape == every[k].shape
            # (without conditioning gradients rows are dealt out otherwise)
            assert float((one[i].double() - every[i].double()).norm()) <= (2 * half(one[i].dtype) + 1e-6) * float(every[i].double().norm())
        assert sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, want=[False] * 8, **kw) == (None,) * 8


def test_gradient_against_differences():
    s = make(12, 24, F32, F32, 3, groups=4, weight=F32, bias=F32, mod=F32, gate=F32, post=True, post_weight=F32, p=0.2)
    kw = keywords(s)
    kept = sds.residual_norm(s["r"], s["h"], keep=True, **kw)[2]
    grads = dict(zip(ORDER, sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, **kw)))

    def loss(**change):
        t = dict(s, **change)
        ref = Norms64(t)
        return float(((ref.n * s["dn"].double()).sum() + (ref.out * s["dr"].double()).sum()).detach())
    for name in ORDER:
        d = torch.randn(s[name].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(len(name)))
        eps = 1e-6
        want = (loss(**{name: s[name].double() + eps * d}) - loss(**{name: s[name].double() - eps * d})) / (2 * eps)
        got = float((grads[name].double() * d).sum())
        assert abs(got - want) <= 1e-5 * float((grads[name].double() * d).abs().sum()) + 1e-6 * abs(want), name


def test_empty_and_shapes():
    x, h = torch.empty(0, 64, device="cuda"), torch.empty(0, 64, device="cuda", dtype=BF16)
    cond = torch.ones(3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    out, n, kept = sds.residual_norm(x, h, gate=cond, scale=cond, shift=cond, weight=w, bias=w, post=True, post_weight=w, keep=True)
    assert out.shape == n.shape == (0, 64) and kept.shape == (0, 8)
    got = sds.residual_norm_backward(n, out, x, h, kept, gate=cond, scale=cond, shift=cond, weight=w, bias=w, post=True, post_weight=w)
    assert all((g == 0).all() for g in got) and got[4].shape == (3, 64)
    r = gen(1)
    x, h, c = r(2, 6, 64), r(2, 6, 64), r(2, 64)
    a = sds.residual_norm(x, h, gate=c)
    b = sds.residual_norm(x.reshape(12, 64), h.reshape(12, 64), gate=c)
    assert a[0].shape == (2, 6, 64) and torch.equal(a[1].reshape(12, 64), b[1])
    assert torch.equal(sds.residual_norm(x, h, gate=c[0])[1], sds.residual_norm(x, h, gate=c[:1])[1])
    stream, n = sds.residual_norm(x)
    assert stream is x or stream.data_ptr() == x.data_ptr()


def test_refusals():
    x, h, w, c = torch.ones(6, 8, device="cuda"), torch.ones(6, 8, device="cuda"), torch.ones(8, device="cuda"), torch.ones(2, 8, device="cuda")
    bad = [lambda: sds.residual_norm(x, h, kind="batch"), lambda: sds.residual_norm(x, h[:3]), lambda: sds.residual_norm(x, h.cpu()), lambda: sds.residual_norm(x, h, weight=w[:4]),
           lambda: sds.residual_norm(x, h, weight=w, bias=w.half()), lambda: sds.residual_norm(x, h, post_weight=w), lambda: sds.residual_norm(x, gate=c),
           lambda: sds.residual_norm(x, post=True), lambda: sds.residual_norm(x, p=0.1), lambda: sds.residual_norm(x, h, gate=torch.ones(4, 8, device="cuda")),
           lambda: sds.residual_norm(x, h, gate=c, scale=c[:1]), lambda: sds.residual_norm(x, h, gate=c, shift=c.half()), lambda: sds.residual_norm(x, h, gate=c[:, :4]),
           lambda: sds.residual_norm(x, h, p=1.5), lambda: sds.residual_norm(x, h, gate=w.expand(6, 8)), lambda: sds.residual_norm(x, stream_out=x),
           lambda: sds.residual_norm(x, h, out=x[:3]), lambda: sds.residual_norm(x.double(), h.double())]
    _, n, kept = sds.residual_norm(x, h, keep=True)
    bad += [lambda: sds.residual_norm_backward(n, x, x, h, kept[:5]), lambda: sds.residual_norm_backward(n[:3], x, x, h, kept), lambda: sds.residual_norm_backward(n, x.half(), x, h, kept),
            lambda: sds.residual_norm_backward(n.half(), x, x, h, kept), lambda: sds.residual_norm_backward(n, x, x, h, kept, want=(True,) * 7),
            lambda: sds.residual_norm_backward(n, x, x, h, kept, workspace=torch.empty(1, device="cuda", dtype=torch.uint8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    long = torch.ones(2, 16385, device="cuda")
    for call, code in ((lambda: sds.residual_norm(long), sb.SDS_EUNSUPPORTED), (lambda: sds.residual_norm(x.bfloat16(), h), sb.SDS_EUNSUPPORTED),
                       (lambda: sds.residual_norm(x, eps=-1.0), sb.SDS_EINVAL), (lambda: sds.residual_norm(x, h, alpha=float("inf")), sb.SDS_EINVAL)):
        with pytest.raises(sds.SdsError) as e:
            call()
        assert e.value.code == code
    with pytest.warns(UserWarning, match="residual_norm records nothing"):
        sds.residual_norm(x, h.clone().requires_grad_(True))


@pytest.mark.parametrize("groups", [1, 8, 48])
def test_captured_step_replays_on_new_inputs(groups):
    opts = dict(groups=groups, weight=F32, bias=F32, mod=BF16, gate=BF16, post=True, post_weight=F32, p=0.1)
    s = make(48, 520, F32, BF16, 30, **opts)
    kw = dict(keywords(s), step=torch.zeros(1, device="cuda", dtype=torch.int32))

    def step():
        out, n, kept = sds.residual_norm(s["r"], s["h"], keep=True, **kw)
        return (out, n) + sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (31, 32):
        new = make(48, 520, F32, BF16, seed, **opts)
        for name in ("r", "h", "dn", "dr", "gate", "scale"):
            s[name].copy_(new[name])
        kw["step"].fill_(seed)
        graph.replay()
        for p, q in zip(out, step()):
            assert torch.equal(p, q)


def test_a_conditioned_block_trains():
    """Linear layers between these norms, with dropout: gradients of a whole block against differentiating it in 64 bits."""
    rows, d, f, groups = 96, 128, 256, 4
    r = gen(77)
    x, cond = r(rows, d), (0.3 * r(groups, 3 * d)).to(BF16)
    w1, w2 = (r(f, d) * d ** -0.5).to(BF16), (r(d, f) * f ** -0.5).to(BF16)
    b1, b2 = 0.1 * r(f), 0.1 * r(d)
    dout, dn_last = r(rows, d), r(rows, d).to(BF16)
    gate, scale, shift = cond[:, :d], cond[:, d:2 * d], cond[:, 2 * d:]
    norm = dict(kind="rms", p=0.1, seed=5, step=2)
    _, n, k0 = sds.residual_norm(x, scale=scale, shift=shift, out_dtype=BF16, keep=True)
    a, k1 = sds.linear(n, w1, b1, "gelu", keep=True)
    h, k2 = sds.linear(a, w2, b2, keep=True)
    out, last, k3 = sds.residual_norm(x, h, gate=gate, keep=True, **norm)
    dx, dh, _, _, _, _, dgate, _ = sds.residual_norm_backward(dn_last, dout, x, h, k3, gate=gate, **norm)
    da, dw2, db2, _ = sds.linear_backward(dh, a, w2, k2, bias=b2)
    dn, dw1, db1, _ = sds.linear_backward(da, n, w1, k1, bias=b1)
    dx, _, _, _, dscale, dshift, _, _ = sds.residual_norm_backward(dn, dx, x, None, k0, scale=scale, shift=shift)
    v = [t.double().requires_grad_(True) for t in (x, w1, b1, w2, b2, gate, scale, shift)]
    spread = lambda t: t.repeat_interleave(rows // groups, 0)  # noqa: E731
    m = xhat64(v[0], "layer", 1e-5) * (1 + spread(v[6])) + spread(v[7])
    q = torch.nn.functional.gelu(m @ v[1].T + v[2]) @ v[3].T + v[4]
    y = v[0] + spread(v[5]) * factor(rows, d, 0.1, 5, 2) * q
    want = torch.autograd.grad([y, xhat64(y, "rms", 1e-5)], v, [dout.double(), dn_last.double()])
    # each of the few tensors between is rounded to bf16 once, independently from element to element
    for got, ref in zip((dx, dw1, db1, dw2, db2, dgate, dscale, dshift), want):
        assert float((got.double() - ref).norm() / ref.norm()) <= 4 * half(BF16)
    assert float((out.double() - y.detach()).norm() / y.detach().norm()) <= half(BF16)
