"""The layer operators on the GPU against their definitions in 64 bits.

Tolerances, derived from the arithmetic. A rounding to type t is off by at most eps_t / 2 relative (h below). Float
sums: a thread adds up to S0 terms one after the other, then a tree of about ten levels, so a sum is off by at most
(S0 + 10) u times the sum of the terms' sizes, u = 2^-24. On the tensor cores a product of 16 terms is added to the
accumulator at a time, with at most one truncation (2 u) per step: (K / 16 + 16) 2 u times the sum of sizes.
"""
import math

import pytest
import torch

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).tiny * torch.finfo(t).eps      # the step of the subnormal range


def close(got, want, bound, what=""):
    """got within half a step of its type of want, and `bound` of error before that rounding."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g = got.double()
    assert torch.isfinite(g).all(), what
    lim = (want.abs() + bound) * half(got.dtype) + bound + tiny(got.dtype)
    over = (g - want).abs() / lim
    assert over.max() <= 1.0, (what, float(over.max()), int(over.argmax()))


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------

TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]
# every thread group of the register kernels at its edges, aligned and not, and rows beyond them
SIZES = [(1, 1), (3, 5), (70, 64), (33, 65), (19, 72), (5, 256), (300, 257), (9, 1000), (301, 1001), (6, 1024), (17, 2048),
         (7, 2049), (4, 4096), (3, 5000), (5, 8192), (6, 16384), (3, 16383), (2, 16385), (3, 20008)]


def plain_norm(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    xhat = (x - mean) * rstd
    wd = torch.ones_like(x[0]) if w is None else w.double()
    bd = torch.zeros_like(x[0]) if b is None else b.double()
    return xhat * wd + bd, mean[..., 0], rstd[..., 0], xhat


def serial(d):
    return max(16, d // 1024 + 1)


def norm_bound(xhat, w, b, d):
    s = (serial(d) + 18) * U
    wd = torch.ones_like(xhat[0]) if w is None else w.double().abs()
    bd = torch.zeros_like(xhat[0]) if b is None else b.double().abs()
    return s * (xhat.abs() + 1.0) * wd + 2 * U * bd


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,d", SIZES)
def test_norm_forward(rows, d, tx, ty):
    r = gen(rows * 1000 + d)
    x = (r(rows, d) * torch.exp(r(rows, 1)) + 3 * r(rows, 1)).to(tx)
    w, b = 1 + 0.3 * r(d), 0.3 * r(d)
    for wt in (F32, ty):
        wv, bv = w.to(wt), b.to(wt)
        y, mean, rstd = sds.layer_norm(x, wv, bv, 1e-5, out_dtype=ty, stats=True)
        want, m, rs, xhat = plain_norm(x, wv, bv, 1e-5)
        close(y, want, norm_bound(xhat, wv, bv, d), (rows, d, tx, ty, wt))
        s = (serial(d) + 18) * U
        assert ((mean.double() - m).abs() <= s * (1 / rs) + U * m.abs()).all()
        assert ((rstd.double() - rs).abs() <= s * rs).all()


def check_norm_grads(got, dy, x, w, eps):
    rows, d = x.shape
    _, _, rs, xhat = plain_norm(x, w, None, eps)
    g, rs = (dy.double() if w is None else dy.double() * w.double()), rs[:, None]
    c2 = (g * xhat).mean(-1, keepdim=True)
    want = rs * (g - g.mean(-1, keepdim=True) - xhat * c2)
    s = 4 * (serial(d) + 18) * U
    size = g.abs() + g.abs().mean(-1, keepdim=True) + (xhat.abs() + 1) * ((g * xhat).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True))
    close(got[0], want, s * rs * size, ("dx", rows, d))
    n = (rows / 148 + min(rows, 888) / 8 + 16) * U + s
    close(got[1], (dy.double() * xhat).sum(0), n * (dy.double().abs() * (xhat.abs() + 1)).sum(0), ("dw", rows, d))
    close(got[2], dy.double().sum(0), n * dy.double().abs().sum(0), ("db", rows, d))


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,d", SIZES + [(5000, 64), (3000, 72), (1999, 1001), (700, 2048), (400, 4096), (333, 8192),
                                            (40, 20001)])
def test_norm_backward(rows, d, tx, ty):
    r = gen(rows * 1000 + d + 1)
    x = (r(rows, d) * torch.exp(0.5 * r(rows, 1)) + r(rows, 1)).to(tx)
    w = (1 + 0.3 * r(d)).to(ty)
    dy = r(rows, d).to(ty)
    _, mean, rstd = sds.layer_norm(x, w, None, 1e-5, out_dtype=ty, stats=True)
    dx, dw, db = sds.layer_norm_backward(dy, x, w, mean, rstd)
    check_norm_grads((dx, dw, db), dy, x, w, 1e-5)


def test_norm_rows_far_from_zero():
    """Rows at 1e4 with a spread of one: what the rounding of the mean costs is taken back out."""
    r = gen(5)
    x = 1e4 + r(64, 2048)
    w, dy = 1 + 0.1 * r(2048), r(64, 2048)
    y, mean, rstd = sds.layer_norm(x, w, None, 0.0, stats=True)
    want, _, rs, xhat = plain_norm(x, w, None, 0.0)
    close(y, want, norm_bound(xhat, w, None, 2048))
    check_norm_grads(sds.layer_norm_backward(dy, x, w, mean, rstd), dy, x, w, 0.0)


@pytest.mark.parametrize("d", [7, 64, 1024, 16384])
def test_norm_special_rows(d):
    """Constant rows give the bias; a NaN or an infinity spoils its own row and no other."""
    r = gen(d)
    x = r(9, d)
    x[0] = 3.25
    x[2, d // 2] = float("nan")
    x[5, d - 1] = float("inf")
    b = r(d)
    y = sds.layer_norm(x, None, b)
    assert torch.equal(y[0], b)
    assert torch.isnan(y[2]).all() and torch.isnan(y[5]).all()
    good = [0, 1, 3, 4, 6, 7, 8]
    want, _, _, xhat = plain_norm(x[good], None, b, 1e-5)
    close(y[good], want, norm_bound(xhat, None, b, d))


@pytest.mark.parametrize("d,pad", [(64, 8), (1000, 3), (2048, 16), (16384, 8), (17000, 1)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_norm_strided_rows_leave_the_rest(d, pad, t):
    """Rows inside a wider buffer: the gaps, and the rows after the last, stay as they were."""
    r = gen(d + pad)
    rows = 11
    xb, yb = r(rows + 2, d + pad).to(t), torch.full((rows + 2, d + pad), 7.0, device="cuda", dtype=t)
    x, y = xb[:rows, :d], yb[:rows, :d]
    if pad % 8:
        x, y = xb[:rows, 1:d + 1], yb[:rows, 1:d + 1]                # an odd start as well
    out = sds.layer_norm(x, out=y)
    assert out.data_ptr() == y.data_ptr()
    want, _, _, xhat = plain_norm(x, None, None, 1e-5)
    close(y, want, norm_bound(xhat, None, None, d))
    y.fill_(7.0)
    assert (yb == 7.0).all()
    _, mean, rstd = sds.layer_norm(x, stats=True)
    # (dy is the constant 7: dx is zero up to its rounding, which the derived bound covers)
    check_norm_grads(sds.layer_norm_backward(y, x, None, mean, rstd), y, x, None, 1e-5)


def test_norm_shapes_and_empty():
    r = gen(3)
    x = r(2, 3, 5, 40)
    y, mean, _ = sds.layer_norm(x, stats=True)
    assert y.shape == x.shape and mean.shape == (2, 3, 5)
    assert torch.equal(y.reshape(30, 40), sds.layer_norm(x.reshape(30, 40)))
    z = x.permute(1, 0, 2, 3)                                        # rows that are not evenly spaced
    with pytest.raises(ValueError):
        sds.layer_norm(z)
    e = torch.empty(0, 40, device="cuda")
    y, mean, rstd = sds.layer_norm(e, stats=True)
    assert y.shape == (0, 40)
    dx, dw, db = sds.layer_norm_backward(e, e, None, mean, rstd)
    assert dx.shape == (0, 40) and (dw == 0).all() and (db == 0).all()
    for bad in (lambda: sds.layer_norm(x, torch.ones(39, device="cuda")), lambda: sds.layer_norm(x.half(), out_dtype=F32),
                lambda: sds.layer_norm(x.double()), lambda: sds.layer_norm(x, torch.ones(40)),
                lambda: sds.layer_norm(x, torch.ones(40, device="cuda"), torch.ones(40, device="cuda", dtype=F16)),
                lambda: sds.layer_norm(x.transpose(-1, -2)), lambda: sds.layer_norm(x, eps=-1.0)):
        with pytest.raises((ValueError, sds.SdsError)):
            bad()


def test_norm_wanted_gradients_and_repeats():
    r = gen(8)
    x, w, dy = r(2000, 1024), r(1024), r(2000, 1024)
    _, mean, rstd = sds.layer_norm(x, w, stats=True)
    full = sds.layer_norm_backward(dy, x, w, mean, rstd)
    for _ in range(3):                                               # fixed order of the sums: same bits
        for p, q in zip(full, sds.layer_norm_backward(dy, x, w, mean, rstd)):
            assert torch.equal(p, q)
    for k in range(3):
        want = [i == k for i in range(3)]
        got = sds.layer_norm_backward(dy, x, w, mean, rstd, want=want)
        for i in range(3):
            assert (got[i] is None) == (i != k)
        assert torch.equal(got[k], full[k])


def test_norm_gradient_against_differences():
    r = gen(9)
    x, w, b, dy = r(5, 96), r(96), r(96), r(5, 96)
    _, mean, rstd = sds.layer_norm(x, w, b, stats=True)
    dx, dw, db = sds.layer_norm_backward(dy, x, w, mean, rstd)
    h = 1e-5
    for v, grad, at in ((r(5, 96), dx, 0), (r(96), dw, 1), (r(96), db, 2)):
        args = [x.double(), w.double(), b.double()]
        step = lambda s: (plain_norm(*[a + (s * h * v.double() if i == at else 0) for i, a in enumerate(args)], 1e-5)[0] * dy.double()).sum()  # noqa: E731,B023
        slope = float((step(1) - step(-1)) / (2 * h))
        # differences are off by h^2 times a third derivative, about 1e-8 here; the float gradient by about 1e-6
        assert abs(slope - float((grad.double() * v.double()).sum())) <= 1e-5 * float((grad.double().abs() * v.double().abs()).sum())


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------


def act64(g, name):
    """act(g) and act'(g) in 64 bits."""
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    p = torch.sigmoid(z)
    return g * p, p + g * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)


class Ffn64:
    """The block in 64 bits, with bounds of the error before each last rounding."""

    def __init__(self, x, wg, wu, wd, act, t):
        x, wg, wu, wd = (v.double() for v in (x, wg, wu, wd))
        self.x, self.wg, self.wu, self.wd, self.t = x, wg, wu, wd, t
        tc = lambda k: (k / 16 + 16) * 2 * U  # noqa: E731
        d, f = x.shape[1], wg.shape[0]
        self.g, self.u = x @ wg.T, x @ wu.T
        eg, eu = tc(d) * (x.abs() @ wg.abs().T), tc(d) * (x.abs() @ wu.abs().T)
        self.a, self.da = act64(self.g, act)
        # fast exponential: a few units of the last place per unit of its argument; 2^-19 covers |g| up to 16
        ap = 2.0 ** -19
        self.ea = self.da.abs() * eg + ap * (self.a.abs() + U) + eg * eg
        self.eda = 2 * eg + ap * (self.da.abs() + 1)                 # |act''| < 2
        self.h = self.a * self.u
        eh = self.ea * (self.u.abs() + eu) + self.a.abs() * eu
        self.eh = eh + half(t) * (self.h.abs() + eh) + tiny(t)       # rounded as an operand
        self.y = self.h @ wd.T
        self.ey = (self.eh + tc(f) * self.h.abs()) @ wd.abs().T
        self.eu, self.tc = eu, tc

    def backward(self, dy):
        dy = dy.double()
        d, f, rows, t, tc = self.x.shape[1], self.wg.shape[0], self.x.shape[0], self.t, self.tc
        dh = dy @ self.wd
        edh = tc(d) * (dy.abs() @ self.wd.abs())
        self.dg, self.du = dh * self.u * self.da, dh * self.a
        edg = edh * (self.u * self.da).abs() + dh.abs() * (self.eu * self.da.abs() + (self.u.abs() + self.eu) * self.eda) + 4 * U * self.dg.abs()
        edu = edh * self.a.abs() + dh.abs() * self.ea + 4 * U * self.du.abs()
        edg = edg + half(t) * (self.dg.abs() + edg) + tiny(t)
        edu = edu + half(t) * (self.du.abs() + edu) + tiny(t)
        self.dx = self.dg @ self.wg + self.du @ self.wu
        self.edx = (edg + tc(2 * f) * self.dg.abs()) @ self.wg.abs() + (edu + tc(2 * f) * self.du.abs()) @ self.wu.abs()
        xa = self.x.abs()
        self.dwg, self.edwg = self.dg.T @ self.x, (edg + tc(rows) * self.dg.abs()).T @ xa
        self.dwu, self.edwu = self.du.T @ self.x, (edu + tc(rows) * self.du.abs()).T @ xa
        self.dwd, self.edwd = dy.T @ self.h, dy.abs().T @ (self.eh + tc(rows) * self.h.abs())


def ffn_inputs(rows, d, f, t, seed):
    r = gen(seed)
    x, wg, wu, wd = r(rows, d), r(f, d) * d ** -0.5, r(f, d) * d ** -0.5, r(d, f) * f ** -0.5
    return [v.to(t) for v in (x, wg, wu, wd, 0.1 * r(rows, d))]


# rows: both forms and their borders; widths: one tile, ragged tiles, a last column block of eight
FFN_SIZES = [(1, 8, 8), (1, 64, 128), (3, 72, 200), (16, 128, 64), (17, 256, 520), (33, 1000, 136), (64, 512, 2048), (100, 136, 1000),
             (128, 264, 392), (129, 64, 64), (200, 8, 72), (300, 520, 1032), (513, 1000, 264), (1100, 256, 1536), (2500, 384, 640)]


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("rows,d,f", FFN_SIZES)
def test_ffn_forward_and_backward(rows, d, f, t):
    act = ("silu", "gelu", "gelu_tanh")[(rows + d) % 3]
    x, wg, wu, wd, dy = ffn_inputs(rows, d, f, t, rows + d + f)
    ref = Ffn64(x, wg, wu, wd, act, t)
    y = sds.gated_ffn(x, wg, wu, wd, act)
    close(y, ref.y, ref.ey, "y")
    y2, kept = sds.gated_ffn(x, wg, wu, wd, act, keep=True)
    assert torch.equal(y, y2)
    got = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)
    ref.backward(dy)
    for name, v in zip(("dx", "dwg", "dwu", "dwd"), got):
        close(v, getattr(ref, name), getattr(ref, "e" + name), name)
    if min(rows, d, f) >= 64:
        # an operand's rounding and the result's, each at most half a step and independent from element to element
        for v, w in zip((y,) + got, (ref.y, ref.dx, ref.dwg, ref.dwu, ref.dwd)):
            assert rel(v, w) <= 2 * half(t)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows", [40, 400])
def test_ffn_activations_over_their_range(act, rows):
    """Pre-activations from -40 to 40: the weights pick single inputs, so that G and U are those inputs."""
    d = f = 128
    eye = torch.eye(d, device="cuda", dtype=BF16)
    x = torch.linspace(-40, 40, rows * d, device="cuda").reshape(d, rows).T.contiguous().to(BF16)
    y, kept = sds.gated_ffn(x, eye, eye, eye, act, keep=True)
    a, da = act64(x.double(), act)
    h = (a * x.double())
    assert ((y.double() - h).abs() <= 2.1 * half(BF16) * h.abs() + 2.0 ** -19 * x.double().abs() + 1e-30).all()
    one = torch.ones_like(x)
    dx, _, _, _ = sds.gated_ffn_backward(one, x, eye, eye, eye, kept)
    dg, du = x.double() * da, a
    want = dg + du
    assert ((dx.double() - want).abs() <= 2.1 * half(BF16) * (dg.abs() + du.abs()) + 2.0 ** -18 * (1 + x.double().abs())).all()


@pytest.mark.parametrize("rows", [5, 300])
def test_ffn_strided_rows_leave_the_rest(rows):
    d, f = 136, 264
    x, wg, wu, wd, dy = ffn_inputs(rows, d, f, BF16, 77)
    wide = torch.full((rows + 3, d + 24), 9.0, device="cuda", dtype=BF16)
    xs = wide.clone()
    xs[:rows, 8:8 + d] = x
    out = wide[:rows, 16:16 + d]
    y, kept = sds.gated_ffn(xs[:rows, 8:8 + d], wg, wu, wd, out=out, keep=True)
    y0, kept0 = sds.gated_ffn(x, wg, wu, wd, keep=True)
    assert torch.equal(y, y0) and y.data_ptr() == out.data_ptr()
    out.fill_(9.0)
    assert (wide == 9.0).all()
    dys = xs.clone()
    dys[:rows, 8:8 + d] = dy
    a = sds.gated_ffn_backward(dys[:rows, 8:8 + d], xs[:rows, 8:8 + d], wg, wu, wd, kept)
    b = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept0)
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_ffn_special_rows_stay_apart():
    """A NaN or an infinity in one row reaches no other row of y and of dx."""
    x, wg, wu, wd, dy = ffn_inputs(300, 128, 256, BF16, 5)
    y, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    dx = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)[0]
    z = x.clone()
    z[7, 3], z[140, 0] = float("nan"), float("inf")
    y2, kept2 = sds.gated_ffn(z, wg, wu, wd, keep=True)
    dx2 = sds.gated_ffn_backward(dy, z, wg, wu, wd, kept2)[0]
    rest = torch.ones(300, dtype=torch.bool, device="cuda")
    rest[7] = rest[140] = False
    assert torch.equal(y[rest], y2[rest]) and torch.equal(dx[rest], dx2[rest])
    assert torch.isnan(y2[7]).all() and not torch.isfinite(y2[140]).any()


def test_ffn_empty_and_refusals():
    x, wg, wu, wd, dy = ffn_inputs(4, 64, 128, BF16, 1)
    y, kept = sds.gated_ffn(x[:0], wg, wu, wd, keep=True)
    assert y.shape == (0, 64)
    dx, dwg, dwu, dwd = sds.gated_ffn_backward(dy[:0], x[:0], wg, wu, wd, kept)
    assert dx.shape == (0, 64) and all((v == 0).all() for v in (dwg, dwu, dwd))
    y, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    for bad in (lambda: sds.gated_ffn(x, wg, wu, wd, "relu"), lambda: sds.gated_ffn(x.float(), wg, wu, wd),
                lambda: sds.gated_ffn(x, wg, wu[:64], wd), lambda: sds.gated_ffn(x, wg, wu, wd.T),
                lambda: sds.gated_ffn(x, wg, wu, wd.half()), lambda: sds.gated_ffn(x[:, :60], wg[:, :60].contiguous(), wu[:, :60].contiguous(), wd[:60].contiguous()),
                lambda: sds.gated_ffn(x, wg.cpu(), wu, wd), lambda: sds.gated_ffn_backward(dy, x, wg, wu, wd, kept[:100]),
                lambda: sds.gated_ffn_backward(dy[:2], x, wg, wu, wd, kept),
                lambda: sds.gated_ffn(x, wg, wu, wd, workspace=torch.empty(8, device="cuda", dtype=torch.uint8))):
        with pytest.raises((ValueError, sds.SdsError)):
            bad()


@pytest.mark.parametrize("rows", [20, 400])
def test_ffn_wanted_gradients_and_repeats(rows):
    x, wg, wu, wd, dy = ffn_inputs(rows, 256, 512, BF16, 2)
    _, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    full = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)
    for p, q in zip(full, sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)):
        assert torch.equal(p, q)
    for want in ([1, 0, 0, 0], [0, 1, 1, 0], [0, 0, 0, 1], [0, 1, 0, 1], [0, 0, 0, 0]):
        got = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept, want=want)
        for k in range(4):
            assert (got[k] is None) == (not want[k])
            assert got[k] is None or torch.equal(got[k], full[k])


def test_ffn_gradient_against_differences():
    x, wg, wu, wd, dy = ffn_inputs(70, 64, 96, F16, 3)
    _, kept = sds.gated_ffn(x, wg, wu, wd, "gelu", keep=True)
    grads = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)
    r = gen(4)
    h = 1e-5
    for at, grad in enumerate(grads):
        v = r(*grad.shape).double()
        args = [a.double() for a in (x, wg, wu, wd)]

        def loss(s):
            p = [a + (s * h * v if i == at else 0) for i, a in enumerate(args)]
            return ((act64(p[0] @ p[1].T, "gelu")[0] * (p[0] @ p[2].T)) @ p[3].T * dy.double()).sum()
        slope = float((loss(1) - loss(-1)) / (2 * h))
        # the gradient's elements are off by about half a step each; differences by about 1e-8
        assert abs(slope - float((grad.double() * v).sum())) <= 3 * half(F16) * float((grad.double() * v).norm()) + 1e-6


# ---------------------------------------------------------------------------------------------
# how they are used together
# ---------------------------------------------------------------------------------------------


def test_residual_block_trains():
    """A pre-norm block r + ffn(norm(r)), forward and backward, as a training step runs it."""
    rows, d, f = 260, 256, 640
    r = gen(11)
    x = r(rows, d)
    w, b = 1 + 0.1 * r(d), 0.1 * r(d)
    wg, wu, wd = ((r(*s) * s[1] ** -0.5).to(BF16) for s in ((f, d), (f, d), (d, f)))
    dy = 0.1 * r(rows, d)
    n, mean, rstd = sds.layer_norm(x, w, b, out_dtype=BF16, stats=True)
    y, kept = sds.gated_ffn(n, wg, wu, wd, keep=True)
    out = x + y.float()
    dn, dwg, dwu, dwd = sds.gated_ffn_backward(dy.to(BF16), n, wg, wu, wd, kept)
    dx, dw, db = sds.layer_norm_backward(dn, x, w, mean, rstd)
    dx = dx + dy
    v = [a.double().requires_grad_(True) for a in (x, w, b, wg, wu, wd)]
    m = v[0].mean(-1, keepdim=True)
    nn = (v[0] - m) / torch.sqrt(((v[0] - m) ** 2).mean(-1, keepdim=True) + 1e-5) * v[1] + v[2]
    o = v[0] + (torch.nn.functional.silu(nn @ v[3].T) * (nn @ v[4].T)) @ v[5].T
    grads = torch.autograd.grad(o, v, dy.double())
    # roundings to bfloat16 along the way: n (reaching G, U and the gradients), h or dG and dU, dy, the results
    assert rel(out, o.detach()) <= 3 * half(BF16)
    for got, want in zip((dx, dw, db, dwg, dwu, dwd), grads):
        assert rel(got, want) <= 4 * half(BF16)


def test_two_streams_at_once():
    """Two calls on different streams, each with workspaces of its own, give what they give alone."""
    a, b = ffn_inputs(600, 256, 1024, BF16, 20), ffn_inputs(90, 512, 768, BF16, 21)
    alone = [sds.gated_ffn(*v[:4]) for v in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for k, v in enumerate((a, b)):
            with torch.cuda.stream(streams[k]):
                got[k].append(sds.gated_ffn(*v[:4]))
                got[k].append(sds.layer_norm(v[0]))
    torch.cuda.synchronize()
    for k, v in enumerate((a, b)):
        for y in got[k][::2]:
            assert torch.equal(y, alone[k])
        for y in got[k][1::2]:
            assert torch.equal(y, sds.layer_norm(v[0]))


@pytest.mark.parametrize("rows", [48, 500])
def test_captured_step_replays_on_new_inputs(rows):
    d, f = 256, 512
    x, wg, wu, wd, dy = ffn_inputs(rows, d, f, BF16, 30)
    w = torch.ones(d, device="cuda")

    def step():
        n, mean, rstd = sds.layer_norm(x, w, None, stats=True)
        y, kept = sds.gated_ffn(n, wg, wu, wd, keep=True)
        g = sds.gated_ffn_backward(dy, n, wg, wu, wd, kept)
        return (y,) + g + sds.layer_norm_backward(g[0], x, w, mean, rstd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (31, 32):
        new = ffn_inputs(rows, d, f, BF16, seed)
        x.copy_(new[0])
        dy.copy_(new[4])
        graph.replay()
        for p, q in zip(out, step()):
            assert torch.equal(p, q)


def test_status_word_of_the_workspace():
    x, wg, wu, wd, _ = ffn_inputs(10, 64, 64, BF16, 40)
    ws = torch.full((sds.gated_ffn_bytes(10, 64, 64).forward_bytes,), 255, device="cuda", dtype=torch.uint8)
    with pytest.raises(sds.SdsError) as e:                           # a word that says a wait gave up
        sds.gated_ffn_status(ws)
    assert e.value.code == sb.SDS_ETIMEOUT
    sds.gated_ffn(x, wg, wu, wd, workspace=ws)
    sds.gated_ffn_status(ws)


def test_capture_of_a_first_call():
    """A process whose first call of an operator is a captured one (nothing is looked up on the device before)."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2501_05370_b200 as sds
torch.manual_seed(0)
x, w = torch.randn(300, 256, device="cuda").bfloat16(), torch.randn(3, 512, 256, device="cuda").bfloat16()
wd = w[2].t().contiguous()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    n, m, r = sds.layer_norm(x, stats=True)
    y, k = sds.gated_ffn(n, w[0], w[1], wd, keep=True)
    d = sds.gated_ffn_backward(y, n, w[0], w[1], wd, k)
    e = sds.layer_norm_backward(d[0], x, None, m, r)
g.replay()
torch.cuda.synchronize()
n, m, r = sds.layer_norm(x, stats=True)
y2, k = sds.gated_ffn(n, w[0], w[1], wd, keep=True)
d2 = sds.gated_ffn_backward(y2, n, w[0], w[1], wd, k)
e2 = sds.layer_norm_backward(d2[0], x, None, m, r)
assert all(torch.equal(a, b) for a, b in zip((y,) + d + e, (y2,) + d2 + e2))
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=root, timeout=240)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_backward_on_two_streams_at_once():
    a, b = ffn_inputs(700, 256, 1024, BF16, 50), ffn_inputs(90, 512, 768, BF16, 51)

    def step(x, wg, wu, wd, dy):
        n, m, r = sds.layer_norm(x, stats=True)
        y, kept = sds.gated_ffn(n, wg, wu, wd, keep=True)
        g = sds.gated_ffn_backward(dy, n, wg, wu, wd, kept)
        return (y,) + g + sds.layer_norm_backward(g[0], x, None, m, r)
    alone = [step(*v) for v in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for k, v in enumerate((a, b)):
            with torch.cuda.stream(streams[k]):
                got[k].append(step(*v))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            assert all(torch.equal(p, q) for p, q in zip(out, alone[k]))


def test_a_call_behind_a_kernel_that_writes_its_inputs():
    """Kernels start beside the end of the kernel in front: what that one writes, weights included, is what they read."""
    x, wg, wu, wd, dy = ffn_inputs(40, 512, 1024, BF16, 60)
    fresh = [ffn_inputs(40, 512, 1024, BF16, 61 + k) for k in range(6)]
    w, b = torch.ones(512, device="cuda"), torch.zeros(512, device="cuda")
    got = []
    for v in fresh:
        for to, src in zip((x, wg, wu, wd, dy), v):
            to.copy_(src)
        w.mul_(1.25)
        n, m, r = sds.layer_norm(x, w, b, stats=True)
        wg.mul_(2.0)
        y, kept = sds.gated_ffn(n, wg, wu, wd, keep=True)
        got.append((y, sds.gated_ffn_backward(dy, n, wg, wu, wd, kept)))
    torch.cuda.synchronize()
    scale = 1.0
    for v, (y, g) in zip(fresh, got):
        scale *= 1.25
        n = sds.layer_norm(v[0], torch.full_like(w, scale), b)
        torch.cuda.synchronize()
        y2, kept = sds.gated_ffn(n, v[1] * 2, v[2], v[3], keep=True)
        assert torch.equal(y, y2)
        assert all(torch.equal(p, q) for p, q in zip(g, sds.gated_ffn_backward(v[4], n, v[1] * 2, v[2], v[3], kept)))


def test_offsets_past_32_bits():
    """More than 2^32 bytes (and 2^31 elements) per array: the last rows are what they are in a small call."""
    rows, d = 140000, 16384
    r = gen(70)
    x = torch.zeros(rows, d, device="cuda", dtype=BF16)
    x[-3:] = r(3, d).to(BF16)
    y, m, rs = sds.layer_norm(x, stats=True)
    want, _, _, xhat = plain_norm(x[-3:], None, None, 1e-5)
    close(y[-3:], want, norm_bound(xhat, None, None, d))
    dy = torch.zeros_like(x)
    dy[-3:] = r(3, d).to(BF16)
    dx = sds.layer_norm_backward(dy, x, None, m, rs, want=(True, False, False))[0]
    small = sds.layer_norm_backward(dy[-3:], x[-3:], None, m[-3:], rs[-3:], want=(True, False, False))[0]
    assert torch.equal(dx[-3:], small) and (dx[:-3] == 0).all()
    del x, y, dy, dx, m, rs
    rows, d, f = 300000, 64, 8192
    x, wg, wu, wd, dy = ffn_inputs(rows, d, f, BF16, 71)
    y, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    dx = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept, want=(1, 0, 0, 0))[0]
    tail = slice(rows - 500, rows)
    ref = Ffn64(x[tail], wg, wu, wd, "silu", BF16)
    close(y[tail], ref.y, ref.ey)
    ref.backward(dy[tail])
    close(dx[tail], ref.dx, ref.edx)


def test_weights_written_by_an_operator_in_front():
    """The second product's kernel asks for its weights before the first one has ended, and must not read them before the
    operator in front of the whole call has written them: here that operator makes every weight in turn."""
    d, f = 1024, 2048
    x, wg, wu, wd, dy = ffn_inputs(8, d, f, BF16, 80)
    raw = [ffn_inputs(8, d, f, BF16, 81 + k)[1:4] for k in range(12)]
    weights = [torch.empty_like(v) for v in (wg, wu, wd)]
    got = []
    for v in raw:
        for which in (2, 0, 1, 2):                 # the forward call comes right behind the one that writes w_down
            sds.layer_norm(v[which], out=weights[which])
        y, kept = sds.gated_ffn(x, *weights, keep=True)
        for which in (2, 0, 1):                    # the gradient call behind the one that writes w_up (the same values)
            sds.layer_norm(v[which], out=weights[which])
        got.append((y,) + sds.gated_ffn_backward(dy, x, *weights, kept))
        for w in weights:
            sds.layer_norm(raw[0][0].reshape(w.shape), out=w)      # (other values again)
    torch.cuda.synchronize()
    for v, out in zip(raw, got):
        normed = [sds.layer_norm(w) for w in v]
        torch.cuda.synchronize()
        y, kept = sds.gated_ffn(x, *normed, keep=True)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, (y,) + sds.gated_ffn_backward(dy, x, *normed, kept)))


def test_a_small_call_behind_a_long_one():
    """A few-row call starts on the SMs that a long call leaves free, and waits there without counting its polls."""
    big = torch.randn(1 << 22, 64, device="cuda").to(BF16)
    w = [torch.randn(64, 64, device="cuda").to(BF16) for _ in range(3)]
    _, kept = sds.gated_ffn(big, *w, keep=True)
    ws = torch.empty(sds.gated_ffn_bytes(1 << 22, 64, 64).backward_bytes, device="cuda", dtype=torch.uint8)
    x, wg, wu, wd, _ = ffn_inputs(4, 512, 1024, BF16, 90)
    want = sds.gated_ffn(x, wg, wu, wd)
    ws2 = torch.empty(sds.gated_ffn_bytes(4, 512, 1024).forward_bytes, device="cuda", dtype=torch.uint8)
    torch.cuda.synchronize()
    sds.gated_ffn_backward(big, big, *w, kept, workspace=ws)
    y = sds.gated_ffn(x, wg, wu, wd, workspace=ws2)
    sds.gated_ffn_status(ws2)
    sds.gated_ffn_status(ws)
    assert torch.equal(y, want)


def test_backward_of_nothing_sets_the_status_word():
    x, wg, wu, wd, dy = ffn_inputs(5, 64, 64, BF16, 95)
    _, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    ws = torch.full((sds.gated_ffn_bytes(5, 64, 64).backward_bytes,), 255, device="cuda", dtype=torch.uint8)
    assert sds.gated_ffn_backward(dy, x, wg, wu, wd, kept, want=(0, 0, 0, 0), workspace=ws) == (None,) * 4
    sds.gated_ffn_status(ws)


# many rows of small layers: the weights' gradients cut their sums over the rows into parts
@pytest.mark.parametrize("rows,d,f,t", [(16421, 64, 128, BF16), (9000, 72, 200, F16), (5000, 1024, 256, BF16), (16384, 256, 512, F16),
                                        (3001, 8, 8, BF16), ((1 << 20) + 5, 64, 64, BF16)])
def test_ffn_gradients_over_many_rows(rows, d, f, t):
    x, wg, wu, wd, dy = ffn_inputs(rows, d, f, t, rows + d)
    y, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    ws = torch.empty(sds.gated_ffn_bytes(rows, d, f).backward_bytes + 4096, device="cuda", dtype=torch.uint8).fill_(77)
    got = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept, workspace=ws)
    assert (ws[-4096:] == 77).all()
    sds.gated_ffn_status(ws)
    ref = Ffn64(x, wg, wu, wd, "silu", t)
    ref.backward(dy)
    for name, v in zip(("dx", "dwg", "dwu", "dwd"), got):
        close(v, getattr(ref, name), getattr(ref, "e" + name), name)
    for want in ((0, 1, 0, 0), (0, 0, 1, 1), (1, 0, 0, 1)):
        for p, q, w in zip(sds.gated_ffn_backward(dy, x, wg, wu, wd, kept, want=want), got, want):
            assert torch.equal(p, q) if w else p is None


def test_capture_behind_two_joined_streams():
    """A captured call with two kernels in front of it, on the capturing stream and on one that it has joined."""
    x, wg, wu, wd, dy = ffn_inputs(48, 256, 512, BF16, 97)
    src = [v.clone() for v in (x, wd)]
    side = torch.cuda.Stream()

    def step():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            wd.copy_(src[1])
            extra = sds.layer_norm(src[0])
        x.copy_(src[0])
        here.wait_stream(side)
        y, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
        side.wait_stream(here)
        with torch.cuda.stream(side):
            g = sds.gated_ffn_backward(dy, x, wg, wu, wd, kept)
        here.wait_stream(side)
        return (sds.layer_norm(y), extra) + g
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        src[0].mul_(-1.5)
        src[1].mul_(0.5)
        x.zero_()
        wd.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        assert all(torch.equal(p, q) for p, q in zip(got, step()))
        torch.cuda.synchronize()


@pytest.mark.parametrize("rows", [7, 700])
def test_output_in_the_place_of_the_input(rows):
    """A row is read before it is written, and x is not read again after the first product."""
    x, wg, wu, wd, _ = ffn_inputs(rows, 256, 512, BF16, 98)
    n, y = sds.layer_norm(x), sds.gated_ffn(x, wg, wu, wd)
    a, b = x.clone(), x.clone()
    assert torch.equal(sds.layer_norm(a, out=a), n) and torch.equal(sds.gated_ffn(b, wg, wu, wd, out=b), y)


def test_most_rows():
    """2^30 rows, the limit, of eight elements (sixteen gigabytes each way)."""
    rows = 1 << 30
    _, wg, wu, wd, _ = ffn_inputs(1, 8, 8, BF16, 99)
    x = torch.zeros(rows, 8, device="cuda", dtype=BF16)
    x[-5:] = gen(99)(5, 8).to(BF16)
    x[12345] = x[-1]
    y = sds.layer_norm(x)
    assert torch.equal(y[-5:], sds.layer_norm(x[-5:])) and torch.equal(y[12345], y[-1]) and int((y[1::4099] != 0).sum()) == 0
    ws = torch.empty(sds.gated_ffn_bytes(rows, 8, 8).forward_bytes, device="cuda", dtype=torch.uint8)
    sds.gated_ffn(x, wg, wu, wd, out=y, workspace=ws)
    sds.gated_ffn_status(ws)
    ref = Ffn64(x[-5:], wg, wu, wd, "silu", BF16)
    close(y[-5:], ref.y, ref.ey)
    assert torch.equal(y[12345], y[-1]) and int((y[1::4099] != 0).sum()) == 0


@pytest.mark.parametrize("rows,d,tx,ty", [(4000, 33, BF16, BF16), (1500, 1, F32, BF16), (2000, 7, F16, F16), (3000, 1001, BF16, BF16),
                                          (2500, 1002, F32, F16), (1300, 3001, F32, F32), (700, 6001, F16, F16), (400, 9001, F32, BF16),
                                          (300, 16383, BF16, BF16)])
def test_norm_backward_of_many_unaligned_rows(rows, d, tx, ty):
    """Rows that share 16-byte vectors with their neighbours, several per group of threads; the array starts at an odd place and
    what lies around it does not matter."""
    r = gen(rows + d)
    flat = torch.full((rows * d + 40,), float("nan"), device="cuda", dtype=tx)
    x = flat[3:3 + rows * d].view(rows, d)
    x.copy_(r(rows, d) + r(rows, 1))
    flat_y = torch.full((rows * d + 40,), float("inf"), device="cuda", dtype=ty)
    dy = flat_y[5:5 + rows * d].view(rows, d)
    dy.copy_(0.1 * r(rows, d))
    w, b = 1 + 0.2 * r(d), 0.2 * r(d)
    _, m, rs = sds.layer_norm(x, w, b, out_dtype=ty, stats=True)
    check_norm_grads(sds.layer_norm_backward(dy, x, w, m, rs), dy, x, w, 1e-5)
