"""Layer norm on as many rows as make every group of threads take several, on the GPU against 64 bits.

Bounds as derived in test_gpu_layers.py: a float sum is off by at most (terms added one after the other + levels of the
tree) 2^-24 of the sum of sizes. A thread adds at most 16 terms of a row one after the other (`serial`), 32 in unaligned rows of
1025 to 4096 columns: 37 additions deep there. They reach the statistics and y by the mean, times <|x - mean|>, which is 0.8 standard
deviations of these normal rows, and halved by rstd: 30 and 19 steps, within the serial + 18 = 34 allowed for either. A column's sum over the
rows adds the rows of a group (at most 14 here), the groups of a CTA (64 / 16 / 8 / 4 / 2 / 1 with the width) and the CTAs' sums (19 and 8,
or 5 and 32): always less than the rows / 148 + min(rows, 888) / 8 + 16 that check_norm_grads allows beside the rows' own error.
"""
import pytest
import torch

import paper_2501_05370_b200 as sds
from test_gpu_layers import F32, TYPES, U, check_norm_grads, close, gen, norm_bound, plain_norm, serial

pytestmark = pytest.mark.gpu

# one per kernel of many rows, with two passes of its groups at least; widths at and beside a kernel's longest row, aligned and not
MANY = [(80000, 64), (80001, 40), (20000, 256), (20003, 72), (9000, 512), (9001, 264), (9000, 1024), (2000, 1024), (5000, 2048), (700, 2048), (2000, 4096),
        (400, 4096), (1500, 8192), (333, 8192), (700, 16384), (457, 8200), (80000, 33), (20000, 255), (9000, 511), (9000, 1001),
        (5000, 2047), (3000, 3001), (1000, 6001), (700, 9001), (500, 16383)]


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,d", MANY)
def test_norm_forward_of_many_rows(rows, d, tx, ty):
    r = gen(rows + d)
    x = (r(rows, d) * torch.exp(r(rows, 1)) + 3 * r(rows, 1)).to(tx)
    w, b = 1 + 0.3 * r(d), 0.3 * r(d)
    for wt in {F32, ty}:
        wv, bv = w.to(wt), b.to(wt)
        want, m, rs, xhat = plain_norm(x, wv, bv, 1e-5)
        y, mean, rstd = sds.layer_norm(x, wv, bv, 1e-5, out_dtype=ty, stats=True)
        close(y, want, norm_bound(xhat, wv, bv, d), (rows, d, tx, ty, wt))
        s = (serial(d) + 18) * U
        assert ((mean.double() - m).abs() <= s * (1 / rs) + U * m.abs()).all()
        assert ((rstd.double() - rs).abs() <= s * rs).all()
        assert torch.equal(y, sds.layer_norm(x, wv, bv, 1e-5, out_dtype=ty))


# more rows per group than its ring holds (four), row counts beside multiples of the groups of a launch; 8200 to 16384 columns: a
# cluster of two CTAs per row, 74 of them
ROUND = [(40000, 64), (12000, 256), (12001, 512), (6000, 1024), (3001, 2048), (1500, 4096), (800, 8192), (512, 16384), (333, 8200), (1021, 12288),
         (75, 16384), (149, 9000), (223, 8208), (445, 16376)]


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,d", ROUND)
def test_norm_backward_of_many_rows(rows, d, tx, ty):
    r = gen(rows + d + 1)
    x = (r(rows, d) * torch.exp(0.5 * r(rows, 1)) + r(rows, 1)).to(tx)
    w = (1 + 0.3 * r(d)).to(ty)
    dy = r(rows, d).to(ty)
    _, mean, rstd = sds.layer_norm(x, w, None, 1e-5, out_dtype=ty, stats=True)
    full = sds.layer_norm_backward(dy, x, w, mean, rstd)
    check_norm_grads(full, dy, x, w, 1e-5)
    for want in ((True, True, True), (True, False, False), (False, True, True)):
        for got, all_, k in zip(sds.layer_norm_backward(dy, x, w, mean, rstd, want=want), full, want):
            assert torch.equal(got, all_) if k else got is None
