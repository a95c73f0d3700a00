"""The linear layer on the GPU against its definition in 64 bits.

Tolerances, derived from the arithmetic. A rounding to type t is off by at most eps_t / 2 relative (half). On the tensor
cores a product of 16 terms is added to the accumulator at a time, with at most one truncation (2 u, u = 2^-24) per
step: (k / 16 + 16) 2 u times the sum of the terms' sizes. Activations are within 2^-19 of themselves and follow the error of their
argument (|act'| < 1.2, |act''| < 2). The kept derivative is a float; dz is rounded to the operands' type before the products.
Sums over rows in float: at most rows / 8 terms one after the other, then a tree.
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
    over = (g - want).abs() / ((want.abs() + bound) * half(got.dtype) + bound + tiny(got.dtype))
    assert over.max() <= 1.0, (what, float(over.max()), int(over.argmax()))


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def act64(g, name):
    """act(g) and act'(g) in 64 bits."""
    if name is None:
        return g, torch.ones_like(g)
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    p = torch.sigmoid(z)
    return g * p, p + g * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)


def tc(k):
    return (k / 16 + 16) * 2 * U


class Linear64:
    """The layer in 64 bits, with bounds of the error before each last rounding."""

    def __init__(self, x, w, b=None, act=None, table=None, step=None, residual=None):
        self.t, self.act, self.step = x.dtype, act, step
        self.x, self.w = x.double(), w.double()
        z = self.x @ self.w.T
        size = self.x.abs() @ self.w.abs().T
        ez = tc(x.shape[1]) * size
        for extra in ([] if b is None else [b.double()]) + ([] if table is None else [table.double()[step.long()]]):
            z = z + extra
            size = size + extra.abs()
            ez = ez + U * size
        a, self.da = act64(z, act)
        ap = 2.0 ** -19 if act else 0.0
        self.ez = ez
        ea = self.da.abs() * ez + ap * (a.abs() + U) + ez * ez if act else ez
        self.y = a if residual is None else a + residual.double()
        self.ey = ea + (0 if residual is None else U * (a.abs() + ea + residual.double().abs()))
        # the derivative as it is kept
        self.eda = 2 * ez + ap * (self.da.abs() + 1) if act else torch.zeros_like(z)
        if act:
            self.eda = self.eda + U * (self.da.abs() + self.eda)
        self.steps = 0 if table is None else table.shape[0]

    def backward(self, dy):
        rows, n = dy.shape
        exact = self.act is None and dy.dtype == self.t
        dy = dy.double()
        dz = dy * self.da
        ez = dy.abs() * self.eda + (0 if self.act is None else U * dz.abs())
        eop = ez if exact else ez + half(self.t) * (dz.abs() + ez) + tiny(self.t)
        self.dx = dz @ self.w
        self.edx = (eop + tc(n) * (dz.abs() + eop)) @ self.w.abs()
        self.dw = dz.T @ self.x
        self.edw = (eop + tc(rows) * (dz.abs() + eop)).T @ self.x.abs()
        s = (rows / 8 + 64) * U
        self.db, self.edb = dz.sum(0), (ez + s * (dz.abs() + ez)).sum(0)
        if self.steps:
            to = lambda v: torch.zeros(self.steps, n, device=v.device, dtype=torch.float64).index_add_(0, self.step.long(), v)  # noqa: E731
            s = (rows + 64) * U
            self.dtable, self.edtable = to(dz), to(ez + s * (dz.abs() + ez))


def inputs(rows, k, n, t, seed, steps=0, ty=None, bias=F32, residual=False):
    r = gen(seed)
    s = dict(x=r(rows, k).to(t), w=(r(n, k) * k ** -0.5).to(t), b=None if bias is None else (0.3 * r(n)).to(bias),
             dy=(0.1 * r(rows, n)).to(ty or t), table=None, step=None, residual=None)
    if steps:
        s["table"] = (0.5 * r(steps, n)).to(t)
        g = torch.Generator(device="cuda").manual_seed(seed)
        s["step"] = torch.randint(0, steps, (rows,), device="cuda", generator=g, dtype=torch.int32)
    if residual:
        s["residual"] = r(rows, n).to(ty or t)
    return s


def check(s, act, ty):
    kw = dict(table=s["table"], step=s["step"])
    ref = Linear64(s["x"], s["w"], s["b"], act, residual=s["residual"], **kw)
    y = sds.linear(s["x"], s["w"], s["b"], act, residual=s["residual"], out_dtype=ty, **kw)
    assert y.dtype == ty
    close(y, ref.y, ref.ey, "y")
    y2, kept = sds.linear(s["x"], s["w"], s["b"], act, residual=s["residual"], out_dtype=ty, keep=True, **kw)
    assert torch.equal(y, y2)
    got = sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], **kw)
    ref.backward(s["dy"])
    close(got[0], ref.dx, ref.edx, "dx")
    close(got[1], ref.dw, ref.edw, "dw")
    if s["b"] is None:
        assert got[2] is None
    else:
        assert got[2].dtype == s["b"].dtype
        close(got[2], ref.db, ref.edb, "db")
    if s["table"] is None:
        assert got[3] is None
    else:
        close(got[3], ref.dtable, ref.edtable, "dtable")
    sds.linear_status()
    return got


# rows: both forms and their borders; widths: one tile, ragged tiles, a last block of any number of columns
SIZES = [(1, 8, 1), (1, 64, 128), (2, 2048, 2048), (3, 72, 201), (16, 128, 64), (17, 256, 519), (33, 1000, 130), (64, 512, 2048), (65, 136, 1000),
         (128, 264, 391), (129, 64, 8), (200, 8, 72), (300, 520, 1033), (513, 1000, 260), (1100, 256, 1536), (2500, 384, 3), (1037, 1000, 2731)]


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_sizes(rows, k, n, t):
    which = rows + k + n
    act = (None, "silu", "gelu", "gelu_tanh")[which % 4]
    ty = t if which % 3 else F32
    bias = (F32, t, None)[(which + rows) % 3]
    check(inputs(rows, k, n, t, which, steps=7 if rows % 2 else 0, ty=ty, bias=bias, residual=which % 2 == 0), act, ty)


@pytest.mark.parametrize("rows,k,n", [(70, 512, 130), (128, 2048, 2048), (256, 2048, 2048), (250, 8192, 640), (500, 4096, 1024), (384, 8192, 2056), (1000, 1024, 1024)])
def test_forms_of_middle_sizes(rows, k, n):
    """Between few rows and many: tiles, and the few-row form with one to eight CTAs along K."""
    check(inputs(rows, k, n, BF16, rows + k, steps=7, residual=True), "silu", BF16)
    check(inputs(rows, k, n, BF16, rows + n, ty=F32, residual=True), None, F32)


@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("ty", [BF16, F32])
@pytest.mark.parametrize("rows,n", [(40, 136), (40, 137), (700, 264), (700, 261)])
def test_every_part_alone_and_together(rows, n, ty, act):
    for bias, steps, residual in ((None, 0, False), (F32, 0, False), (None, 5, False), (None, 0, True), (BF16, 5, True)):
        check(inputs(rows, 192, n, BF16, rows + n, steps=steps, ty=ty, bias=bias, residual=residual), act, ty)


@pytest.mark.parametrize("rows", [50, 600])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_over_their_range(act, rows):
    """z is x itself: from far below to far above, where the activation is 0 or its argument."""
    k = 64
    v = torch.linspace(-30, 30, rows * k, device="cuda").reshape(rows, k).to(F16)
    eye = torch.eye(k, device="cuda", dtype=F16)
    y, kept = sds.linear(v, eye, None, act, keep=True, out_dtype=F32)
    a, da = act64(v.double(), act)
    # float's exponential is off by a few units per unit of its argument, up to |g| = 30
    assert ((y.double() - a).abs() <= 2.0 ** -18 * a.abs() + 2.0 ** -30).all()
    dx = sds.linear_backward(torch.ones_like(v), v, eye, kept)[0]
    assert ((dx.double() - da).abs() <= (2 * half(F16) + 2.0 ** -17) * da.abs() + 2 * tiny(F16) + 2.0 ** -22).all()


@pytest.mark.parametrize("rows,k,n", [(5, 64, 72), (300, 64, 72), (300, 72, 133)])
def test_strided_rows_leave_the_rest(rows, k, n):
    r = gen(rows + n)
    big = r(rows, k + 16).to(BF16)
    x = big[:, 8:8 + k]
    w = (r(n, k) * 0.1).to(BF16)
    res = r(rows, n + 5)[:, 1:1 + n]
    out = torch.full((rows, n + 7), 7.0, device="cuda")
    y = sds.linear(x, w, None, "silu", residual=res, out_dtype=F32, out=out[:, 3:3 + n])
    ref = Linear64(x, w, None, "silu", residual=res)
    close(y, ref.y, ref.ey, "y")
    assert (out[:, :3] == 7).all() and (out[:, 3 + n:] == 7).all()
    # a batch of positions, every second one
    x3 = big.reshape(1, rows, k + 16)[:, :, 8:8 + k].expand(1, rows, k)
    assert torch.equal(sds.linear(x3, w, None, "silu")[0], sds.linear(x, w, None, "silu"))
    dy = r(rows, n + 3)[:, 1:1 + n].to(BF16)
    kept = sds.linear(x, w, None, None, keep=True)[1]
    ref = Linear64(x, w)
    ref.backward(dy)
    dx, dw, _, _ = sds.linear_backward(dy, x, w, kept)
    close(dx, ref.dx, ref.edx, "dx")
    close(dw, ref.dw, ref.edw, "dw")


def test_output_in_the_place_of_the_residual():
    for rows in (7, 500):
        for ty in (F32, BF16):
            for n in (128, 77):
                s = inputs(rows, 128, n, BF16, rows, ty=ty, residual=True)
                want = sds.linear(s["x"], s["w"], s["b"], "silu", residual=s["residual"], out_dtype=ty)
                got = sds.linear(s["x"], s["w"], s["b"], "silu", residual=s["residual"], out_dtype=ty, out=s["residual"])
                assert got.data_ptr() == s["residual"].data_ptr() and torch.equal(got, want)


@pytest.mark.parametrize("rows,n", [(40, 64), (500, 64), (500, 67)])
def test_steps_outside_the_table(rows, n):
    s = inputs(rows, 64, n, BF16, 3, steps=6)
    bad = s["step"].clone()
    bad[3], bad[rows - 1] = 6, -1
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[3] = rest[rows - 1] = False
    y, kept = sds.linear(s["x"], s["w"], s["b"], "silu", table=s["table"], step=bad, keep=True)
    good, _ = sds.linear(s["x"], s["w"], s["b"], "silu", table=s["table"], step=s["step"], keep=True)
    assert torch.isnan(y[~rest]).all() and torch.equal(y[rest], good[rest])
    got = sds.linear_backward(s["dy"], s["x"], s["w"], kept, table=s["table"], step=bad)
    ref = Linear64(s["x"][rest], s["w"], s["b"], "silu", table=s["table"], step=s["step"][rest])
    ref.backward(s["dy"][rest])
    close(got[3], ref.dtable, ref.edtable, "dtable")


@pytest.mark.parametrize("rows,n,steps,how", [(5000, 72, 250, "even"), (5000, 264, 3, "even"), (4097, 100, 1, "even"), (3000, 64, 1000, "few"),
                                              (5000, 520, 40, "skewed"), (333, 2048, 65535, "even"), (32, 64, 4, "ordered"),
                                              (64, 64, 2, "ordered"), (40000, 16, 5, "ordered")])
def test_gradient_of_the_table(rows, n, steps, how):
    """Runs of one step that fill a slice, cross several, begin or end at its border; steps without rows."""
    s = inputs(rows, 64, n, BF16, rows + n, steps=steps)
    g = torch.Generator(device="cuda").manual_seed(1)
    if how == "few":
        s["step"] = torch.randint(0, 5, (rows,), device="cuda", generator=g, dtype=torch.int32) * 7 + 3
    elif how == "skewed":
        s["step"] = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.9, 11, s["step"]).int()
    elif how == "ordered":
        s["step"] = (torch.arange(rows, device="cuda") * steps // rows).int()
    kw = dict(table=s["table"], step=s["step"])
    for act in ("silu", None):
        kept = sds.linear(s["x"], s["w"], s["b"], act, keep=True, **kw)[1]
        ref = Linear64(s["x"], s["w"], s["b"], act, **kw)
        ref.backward(s["dy"])
        first = sds.linear_backward(s["dy"], s["x"], s["w"], kept, want=(False, False, False, True), **kw)
        assert first[:3] == (None, None, None)
        close(first[3], ref.dtable, ref.edtable, "dtable")
        again = sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], **kw)
        assert torch.equal(first[3], again[3])


@pytest.mark.parametrize("rows,k,n,t", [(16421, 64, 128, BF16), (9000, 72, 200, F16), (5000, 1024, 256, BF16), (16384, 256, 512, F16), (4000, 8, 5, BF16)])
def test_gradients_over_many_rows(rows, k, n, t):
    got = check(inputs(rows, k, n, t, 5, steps=10), "silu", t)
    assert all(torch.equal(a, b) for a, b in zip(got, check(inputs(rows, k, n, t, 5, steps=10), "silu", t)))


@pytest.mark.parametrize("rows,k,n", [(64, 8192, 2048), (100, 8192, 264), (700, 1024, 512), (700, 8192, 512), (3000, 8192, 520), (3000, 2000, 519)])
def test_long_sums_of_float_results(rows, k, n):
    """The tensor cores truncate as they add: at most 60 additions (960 products) are left to one accumulator where the result is a float. One
    loses 2^-24 of the running sum on average, which is two thirds of the final one on average: 60 * 2^-24 * 2 / 3 of it, and float's own
    roundings. (512 additions at k = 8192 would lose 2e-5.)"""
    s = inputs(rows, k, n, BF16, 3, ty=F32, residual=True)
    want = s["x"].double() @ s["w"].double().T
    y = sds.linear(s["x"], s["w"], out_dtype=F32)
    assert float((y.double() - want).norm() / want.norm()) <= 60 * 2 * U / 3 + 4 * U
    y = sds.linear(s["x"], s["w"], residual=s["residual"], out_dtype=F32)
    want = want + s["residual"].double()
    assert float((y.double() - want).norm() / want.norm()) <= 60 * 2 * U / 3 + 4 * U


def test_gradient_against_differences():
    r = gen(9)
    x, w, b, table = r(40, 24).to(F16), (0.3 * r(48, 24)).to(F16), 0.2 * r(48), (0.4 * r(5, 48)).to(F16)
    step = torch.arange(40, device="cuda", dtype=torch.int32) % 5
    dy = r(40, 48)
    for act in ("silu", "gelu", "gelu_tanh"):
        kept = sds.linear(x, w, b, act, table=table, step=step, keep=True)[1]
        grads = sds.linear_backward(dy, x, w, kept, bias=b, table=table, step=step)

        def loss(x, w, b, table):
            y = act64(x @ w.T + b + table[step.long()], act)[0]
            return float((y * dy.double()).sum())
        v = [q.double() for q in (x, w, b, table)]
        for i in range(4):
            d = torch.randn(v[i].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i), dtype=torch.float64)
            eps = 1e-5
            up, down = [list(v), list(v)]
            up[i], down[i] = v[i] + eps * d, v[i] - eps * d
            want = (loss(*up) - loss(*down)) / (2 * eps)
            got = float((grads[i].double() * d).sum())
            # every element's gradient is within three roundings of f16 (dz, act', the result) of itself: in sum, of the sum of sizes
            size = float((grads[i].double() * d).abs().sum())
            assert abs(got - want) <= 4 * half(F16) * size * 4 + 1e-5 * abs(want)


def test_many_rows_with_a_table():
    """More slices of the list than a grid's second dimension has."""
    rows, n, steps = 8_500_000, 8, 3
    s = inputs(rows, 8, n, BF16, 5, steps=steps)
    kw = dict(table=s["table"], step=s["step"])
    kept = sds.linear(s["x"], s["w"], s["b"], None, keep=True, **kw)[1]
    _, _, db, dt = sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], want=(False, False, True, True), **kw)
    dy = s["dy"].double()
    want = torch.stack([dy[s["step"] == i].sum(0) for i in range(steps)])
    size = torch.stack([dy[s["step"] == i].abs().sum(0) for i in range(steps)])
    # slices of 32 rows, joined eight at a time in one chain of rows / 256, or (bias) parts of 128 in chains of rows / 1024
    close(dt, want, (rows / 256 + 64) * U * size, "dtable")
    close(db, dy.sum(0), (rows / 1024 + 64) * U * dy.abs().sum(0), "db")
    big = torch.empty(1 << 21, 8, device="cuda", dtype=BF16)
    with pytest.raises(sds.SdsError) as e:
        sds.linear_backward(big, big, s["w"], sds.linear(big[:1], s["w"], keep=True)[1], table=torch.empty(40000, 8, device="cuda", dtype=BF16),
                            step=torch.zeros(1 << 21, device="cuda", dtype=torch.int32))
    assert e.value.code == sb.SDS_EUNSUPPORTED


def test_empty_and_shapes():
    w, b, table = torch.randn(16, 8, device="cuda").bfloat16(), torch.randn(16, device="cuda"), torch.randn(3, 16, device="cuda").bfloat16()
    x = torch.empty(2, 0, 8, device="cuda", dtype=BF16)
    step = torch.empty(0, device="cuda", dtype=torch.int32)
    y, kept = sds.linear(x, w, b, "silu", table=table, step=step, keep=True)
    assert y.shape == (2, 0, 16)
    dx, dw, db, dt = sds.linear_backward(y, x, w, kept, bias=b, table=table, step=step)
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all() and (dt == 0).all() and dt.shape == table.shape
    x = torch.randn(3, 4, 8, device="cuda").bfloat16()
    y = sds.linear(x, w, b)
    assert y.shape == (3, 4, 16) and torch.equal(y.reshape(12, 16), sds.linear(x.reshape(12, 8), w, b))
    assert sds.linear(x[0, 0], w).shape == (16,)


def test_special_rows_stay_apart():
    for rows in (20, 400):
        s = inputs(rows, 64, 72, BF16, 11)
        want = sds.linear(s["x"], s["w"], s["b"], "gelu")
        x = s["x"].clone()
        x[3, 5], x[7, 0] = float("inf"), float("nan")
        y = sds.linear(x, s["w"], s["b"], "gelu")
        rest = [i for i in range(rows) if i not in (3, 7)]
        assert torch.equal(y[rest], want[rest]) and torch.isnan(y[7]).all() and not torch.isfinite(y[3]).all()


def test_refusals():
    x, w = torch.randn(4, 64, device="cuda").bfloat16(), torch.randn(24, 64, device="cuda").bfloat16()
    b, table, step = torch.randn(24, device="cuda"), torch.randn(3, 24, device="cuda").bfloat16(), torch.zeros(4, device="cuda", dtype=torch.int32)
    bad = [lambda: sds.linear(x, w, b, "relu"), lambda: sds.linear(x.float(), w), lambda: sds.linear(x, w.half()), lambda: sds.linear(x, w[:, :32]),
           lambda: sds.linear(x, w.t()), lambda: sds.linear(x, w, b[:8]), lambda: sds.linear(x, w, b, table=table), lambda: sds.linear(x, w, b, step=step),
           lambda: sds.linear(x, w, table=table.float(), step=step), lambda: sds.linear(x, w, table=table, step=step.long()),
           lambda: sds.linear(x, w, table=table, step=step[:3]), lambda: sds.linear(x, w, residual=torch.zeros(4, 24, device="cuda")),
           lambda: sds.linear(x, w, residual=torch.zeros(4, 64, device="cuda", dtype=BF16)), lambda: sds.linear(x, w.cpu()),
           lambda: sds.linear(x, w, out=torch.zeros(4, 64, device="cuda", dtype=BF16)), lambda: sds.linear(x.double(), w.double()),
           lambda: sds.linear(x, w, workspace=torch.empty(8, device="cuda", dtype=torch.uint8)), lambda: sds.linear(x, w, b.double())]
    y, kept = sds.linear(x, w, b, "silu", keep=True)
    bad += [lambda: sds.linear_backward(x, x, w, kept), lambda: sds.linear_backward(y, x, w, kept[:-256]), lambda: sds.linear_backward(y, x, w, None),
            lambda: sds.linear_backward(y, x, w, kept, want=(True,))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    odd = torch.randn(4, 63, device="cuda").bfloat16()
    for call in (lambda: sds.linear(odd, torch.randn(24, 63, device="cuda").bfloat16()), lambda: sds.linear(x, w, out_dtype=F16),
                 lambda: sds.linear(torch.randn(4, 65, device="cuda").bfloat16()[:, 1:], w)):
        with pytest.raises(sds.SdsError) as e:
            call()
        assert e.value.code == sb.SDS_EUNSUPPORTED
    with pytest.warns(UserWarning, match="linear records nothing"):
        sds.linear(x, w.clone().requires_grad_(True))


@pytest.mark.parametrize("rows", [48, 500])
def test_captured_step_replays_on_new_inputs(rows):
    s = inputs(rows, 256, 520, BF16, 30, steps=9)

    def step():
        y, kept = sds.linear(s["x"], s["w"], s["b"], "gelu", table=s["table"], step=s["step"], keep=True)
        return (y,) + sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], table=s["table"], step=s["step"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (31, 32):
        new = inputs(rows, 256, 520, BF16, seed, steps=9)
        for name in ("x", "dy", "step"):
            s[name].copy_(new[name])
        graph.replay()
        for p, q in zip(out, step()):
            assert torch.equal(p, q)


def test_two_streams_at_once():
    a, b = inputs(500, 256, 520, BF16, 1, steps=4), inputs(60, 512, 260, F16, 2, steps=4)

    def step(s):
        kw = dict(table=s["table"], step=s["step"])
        y, kept = sds.linear(s["x"], s["w"], s["b"], "silu", keep=True, **kw)
        return (y,) + sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], **kw)
    want = step(a), step(b)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [[], []]
    for _ in range(10):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                outs[i].append(step(s))
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert all(torch.equal(p, q) for p, q in zip(o, want[i]))


def test_layers_of_the_mlp_denoiser():
    """A stack of these layers is the sampler's MLP denoiser: the same network through sds_denoise."""
    import numpy as np
    import workloads as wl
    w = wl.WORKLOADS["cfg3"].scaled(d=256, B=160, L=1, K=6, mlp_dims=[256, 384, 256])
    mp = w.mlp_params()
    s = sds.sampler_for(w, mlp=mp)
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.standard_normal((160, 256)).astype(np.float32)).cuda()
    k = torch.from_numpy(rng.integers(0, 6, size=160).astype(np.int32)).cuda()
    want = s.denoise(x, k)
    s.close()
    bits = lambda v: torch.from_numpy(np.ascontiguousarray(v).view(np.int16)).cuda().view(BF16)  # noqa: E731
    h = x.to(BF16)
    for i, wt in enumerate(mp.weights):
        last = i == len(mp.weights) - 1
        b = torch.from_numpy(np.asarray(mp.bias[i], np.float32)).cuda()
        if last:
            h = sds.linear(h, bits(wt), b, out_dtype=F32)
        else:
            h = sds.linear(h, bits(wt), b, "silu", table=bits(mp.temb[i]), step=k)
    # the same operands and sums in another order: a hidden value may round the other way (2^-8 of it), and few do
    assert float((h - want).norm() / want.norm()) <= 2.0 ** -8
