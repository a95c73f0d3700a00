"""Numbers among the arguments of dropout and the residual norm: integers of any kind are taken, what is no number or out of range is a ValueError."""
import numpy as np
import pytest
import torch

import paper_2501_05370_b200 as sds

pytestmark = pytest.mark.gpu


def test_integers_of_any_kind():
    x = torch.ones(4, 64, device="cuda")
    want = sds.dropout(x, 0.5, 7, 3, row0=2)
    for kind in (np.int64, np.uint32, np.int32, np.uint64):
        assert torch.equal(sds.dropout(x, np.float64(0.5), kind(7), kind(3), row0=kind(2)), want)
        assert torch.equal(sds.residual_norm(torch.zeros_like(x), x, p=np.float32(0.5), seed=kind(7), step=kind(3), row0=kind(2))[0], want)
    last = 2 ** 64 - 1
    assert torch.equal(sds.dropout(x, 0.5, last), sds.dropout(x, 0.5, np.uint64(last)))


@pytest.mark.parametrize("kw", [dict(step=1 << 70), dict(step=-(1 << 70)), dict(step=1.5), dict(step="3"), dict(row0=1 << 63), dict(row0=1 << 70), dict(row0=None),
                                dict(seed=1 << 70), dict(seed=-1), dict(seed=np.int64(-1)), dict(seed=2.0), dict(seed="7"), dict(p="0.1"), dict(p=None),
                                dict(p=10 ** 400)])
def test_what_is_no_number_or_out_of_range(kw):
    x = torch.ones(4, 64, device="cuda")
    args = dict(dict(p=0.5, seed=7), **kw)
    n, kept = sds.residual_norm(x, x, keep=True)[1:]
    for call in (lambda: sds.dropout(x, **args), lambda: sds.dropout_backward(x, **args), lambda: sds.residual_norm(x, x, **args),
                 lambda: sds.residual_norm_backward(n, None, x, x, kept, **args)):
        with pytest.raises(ValueError):
            call()


def test_alpha_and_eps():
    x = torch.ones(4, 64, device="cuda")
    for kw in (dict(alpha="1"), dict(alpha=None), dict(eps="1e-5"), dict(eps=10 ** 400)):
        with pytest.raises(ValueError):
            sds.residual_norm(x, x, **kw)
