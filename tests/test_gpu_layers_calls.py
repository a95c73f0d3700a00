"""How the layer operators are called, on the GPU: reports of waits that gave up, errors, warnings, host threads."""
import threading

import pytest
import torch

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb
from test_gpu_layers import BF16, ffn_inputs

pytestmark = pytest.mark.gpu


def test_a_wait_that_gave_up_is_reported_without_a_workspace():
    """A wait that runs out (after 200 polls, on a barrier nobody arrives on) sets the call's status word and the device's, which
    says so once; the context stays usable."""
    x, wg, wu, wd, _ = ffn_inputs(10, 64, 64, BF16, 40)
    want = sds.gated_ffn(x, wg, wu, wd)
    sds.gated_ffn_status()
    ws = torch.full((sds.gated_ffn_bytes(10, 64, 64).forward_bytes,), 255, device="cuda", dtype=torch.uint8)
    stream = torch.cuda.current_stream().cuda_stream
    assert sds.load().sds_selftest_gated_ffn_wait(200, ws.data_ptr(), stream) == sb.SDS_OK
    with pytest.raises(sds.SdsError) as e:
        sds.gated_ffn_status(ws)
    assert e.value.code == sb.SDS_ETIMEOUT
    assert torch.equal(sds.gated_ffn(x, wg, wu, wd, workspace=ws), want)      # (the next call's own word says nothing)
    sds.gated_ffn_status(ws)
    with pytest.raises(sds.SdsError) as e:
        sds.gated_ffn_status()
    assert e.value.code == sb.SDS_ETIMEOUT
    sds.gated_ffn_status()
    assert torch.equal(sds.gated_ffn(x, wg, wu, wd), want)
    sds.gated_ffn_status()


def test_out_of_memory_is_torchs_error():
    """What a call allocates and cannot get (11 TB of kept state, 2 TB of workspace) raises as torch's own allocations do; the next
    call runs."""
    x, wg, wu, wd, _ = ffn_inputs(1 << 20, 8, 1 << 20, BF16, 41)
    for keep in (True, False):
        with pytest.raises(torch.OutOfMemoryError) as e:
            sds.gated_ffn(x, wg, wu, wd, keep=keep)
        assert "C++" not in str(e.value) and "frame #" not in str(e.value)
    y = sds.gated_ffn(x[:3], wg[:64].contiguous(), wu[:64].contiguous(), wd[:, :64].contiguous())
    assert torch.isfinite(y).all()
