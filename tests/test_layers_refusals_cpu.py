"""Further refusals of the layer operators and their denoiser, answered on the host before any launch (no GPU needed; device
pointers are numbers that nothing reads)."""
import ctypes as C

import numpy as np
import pytest

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb


@pytest.mark.parametrize("shift,code", [(0, sb.SDS_OK), (4, sb.SDS_OK), (1, sb.SDS_EINVAL), (2, sb.SDS_EINVAL)])
@pytest.mark.parametrize("at", [0, 1, 2, 3])
def test_gated_denoiser_norm_vectors_are_floats(at, shift, code):
    """Weight and bias of a block's norm are read as floats: 4-byte aligned, or refused as sds_layer_norm refuses them."""
    nblock, d, f = 2, 64, 128
    W = (C.c_void_p * (3 * nblock))(*[0x100000 + 0x1000 * i for i in range(3 * nblock)])
    norm = (C.c_void_p * (2 * nblock))(*[0x200000 + 0x1000 * i + (shift if i == at else 0) for i in range(2 * nblock)])
    temb = (C.c_void_p * nblock)(*([None] * nblock))
    dims = (C.c_int32 * 3)(d, f, sb.SDS_ACT_SILU)
    den = sb.SdsDenoiser()
    den.kind, den.nlayer = sb.SDS_DEN_GATED, nblock
    den.W_dev, den.bias_dev, den.temb_dev, den.dims = (C.cast(v, C.c_void_p) for v in (W, norm, temb, dims))
    a = np.full(5, 0.5, np.float32)
    sch = sb.SdsSchedule(5, a.ctypes.data, a.ctypes.data, a.ctypes.data, None, 0)
    n = C.c_size_t(0)
    assert sds.load().sds_workspace_bytes(C.byref(sch), C.byref(den), 8, d, 4, C.byref(n)) == code


def test_report_of_a_wait_that_gave_up_checks_its_arguments():
    f = sds.load().sds_selftest_gated_ffn_wait
    for polls, ws in ((0, 0x10000), (-1, 0x10000), ((1 << 16) + 1, 0x10000), (10, None), (10, 0x10010)):
        assert f(polls, ws, None) == sb.SDS_EINVAL
