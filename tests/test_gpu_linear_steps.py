"""Rows of the linear layer whose step is outside the table (a padded batch): NaN forward, and no part in any gradient.

Bounds as in test_gpu_linear.py, over the rows that are left.
"""
import pytest
import torch
from test_gpu_linear import Linear64, close, inputs

import paper_2501_05370_b200 as sds

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
WANT = [(True, True, True, True), (True, True, True, False), (False, False, True, False), (True, False, False, False), (False, True, False, True)]


@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("t,ty", [(BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("rows,n", [(9, 64), (40, 67), (500, 64), (500, 133), (3000, 512)])
@pytest.mark.parametrize("special", [False, True])
def test_rows_outside_the_table_take_no_part(rows, n, t, ty, act, special):
    s = inputs(rows, 72, n, t, rows + n, steps=6, ty=ty)
    out = torch.zeros(rows, dtype=torch.bool, device="cuda")
    out[torch.tensor([0, 3, rows // 2, rows // 2 + 1, rows - 1], device="cuda")] = True
    step = s["step"].clone()
    step[out] = torch.tensor([6, -1, 2 ** 31 - 1, -2 ** 31, 7], device="cuda", dtype=torch.int32)[:int(out.sum())]
    kw = dict(table=s["table"], step=step)
    y, kept = sds.linear(s["x"], s["w"], s["b"], act, out_dtype=ty, keep=True, **kw)
    assert torch.isnan(y[out]).all() and torch.isfinite(y[~out]).all()
    dy = s["dy"].clone()
    if special:                                                  # as the gradient of what came from a NaN
        dy[out] = float("nan")
        dy[0] = float("inf")
    ref = Linear64(s["x"][~out], s["w"], s["b"], act, table=s["table"], step=step[~out])
    ref.backward(s["dy"][~out])
    for want in WANT:
        dx, dw, db, dtable = sds.linear_backward(dy, s["x"], s["w"], kept, bias=s["b"], want=want, **kw)
        assert tuple(g is not None for g in (dx, dw, db, dtable)) == want
        if dx is not None:
            assert (dx[out] == 0).all()
            close(dx[~out], ref.dx, ref.edx, "dx")
        for g, value, bound, name in ((dw, ref.dw, ref.edw, "dw"), (db, ref.db, ref.edb, "db"), (dtable, ref.dtable, ref.edtable, "dtable")):
            if g is not None:
                close(g, value, bound, name)


def test_every_row_outside():
    s = inputs(300, 64, 72, BF16, 1, steps=3)
    step = torch.full((300,), -1, device="cuda", dtype=torch.int32)
    for act in (None, "gelu"):
        y, kept = sds.linear(s["x"], s["w"], s["b"], act, table=s["table"], step=step, keep=True)
        assert torch.isnan(y).all()
        assert all((g == 0).all() for g in sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], table=s["table"], step=step))
