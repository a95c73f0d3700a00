"""Rows and elements of the residual norm at which sums cancel or a mask hides what is not finite.

u = 2^-24. A sum of terms of one sign: at most 24 additions one behind the other (eight columns of a thread, five steps in a warp, the
warps' sums), so it is within 24 u of itself, and the mean, behind 1 / d and its product, within 26 u.
"""
import pytest
import torch

import paper_2501_05370_b200 as sds

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


@pytest.mark.parametrize("d", [7, 64, 300, 1001, 2048, 4096, 4104, 5001, 8192, 9000, 15072, 16384])
@pytest.mark.parametrize("eps", [1e-12, 1e-5])
def test_constant_rows_far_from_zero(d, eps):
    """xhat is 0, up to what is left of the mean: v = c - mean is exact and at most 26 u c, the mean of v is within 26 u of it, and the
    product with 1 / sqrt(variance + eps), at most 1 / sqrt(eps), rounds v's share once more: (26 * 26 + 26 + 2) u^2 c / sqrt(eps)."""
    rows = 400
    c = 10.0 ** torch.linspace(0, 5, rows, device="cuda")[:, None]
    x = c.expand(rows, d).contiguous()
    zero, w = torch.zeros_like(x), 1.0 + 0.1 * gen(d)(d)
    bound = (26 * 26 + 28) * U * U * c.double() / eps ** 0.5
    dn = gen(d + 1)(rows, d)
    for post in (False, True):
        r, h = (zero, x) if post else (x, zero)
        out, n, kept = sds.residual_norm(r, h, post=post, eps=eps, keep=True)
        assert torch.isfinite(n).all()
        if post:
            assert (out.double().abs() <= bound * (1 + 4 * U)).all()
        else:
            assert torch.equal(out, x) and (n.double().abs() <= bound).all()
        grads = sds.residual_norm_backward(dn, None, r, h, kept, post=post, weight=w)
        assert all(g is None or torch.isfinite(g).all() for g in grads)


@pytest.mark.parametrize("tr,th", [(F32, F32), (F32, BF16), (F16, F16)])
@pytest.mark.parametrize("rows,d,groups", [(24, 40, 1), (24, 40, 24), (24, 40, 4), (300, 1000, 1), (300, 1000, 300), (300, 1000, 6), (40, 131, 8), (40, 131, 40),
                                           (20, 6000, 5), (20, 16384, 1)])
@pytest.mark.parametrize("cond", ["gate", "gate scale shift", ""])
def test_what_is_dropped_may_be_anything(rows, d, groups, cond, tr, th):
    """A dropped element of h adds nothing, whatever it is: every result and gradient is that of zeros in its place."""
    g = gen(rows + d)
    r, h = g(rows, d).to(tr), g(rows, d).to(th)
    kw = {name: (0.5 * g(groups, d)).to(th) for name in cond.split()}
    kw.update(weight=1.0 + 0.1 * g(d), p=0.3, seed=11, step=2)
    dropped = sds.dropout(torch.ones(rows, d, device="cuda"), 0.3, 11, 2) == 0
    zeros, bad = h.clone(), h.clone()
    zeros[dropped] = 0.0
    values = torch.tensor([float("inf"), float("-inf"), float("nan")], device="cuda", dtype=th)
    bad[dropped] = values[torch.arange(int(dropped.sum()), device="cuda") % 3]
    dn, dr = g(rows, d).to(th), g(rows, d).to(tr)
    results = []
    for v in (zeros, bad):
        out, n, kept = sds.residual_norm(r, v, keep=True, **kw)
        results.append((out, n) + sds.residual_norm_backward(dn, dr, r, v, kept, **kw))
    for i, (a, b) in enumerate(zip(*results)):
        assert a is None and b is None or torch.equal(a, b) and torch.isfinite(b).all(), i
