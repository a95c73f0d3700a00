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


def test_a_call_that_drops_a_gradient_says_so():
    """Nothing is recorded for autograd. Where torch would record something, a forward call warns; its values stay the same."""
    import warnings
    x, wg, wu, wd, dy = ffn_inputs(9, 64, 64, BF16, 42)
    w = torch.ones(64, device="cuda")
    norm = lambda x, w: sds.layer_norm(x, w)  # noqa: E731
    block = lambda x, w: sds.gated_ffn(x, wg, w, wd)  # noqa: E731
    leaf = lambda v: v.clone().requires_grad_(True)  # noqa: E731
    for call, v in ((norm, w), (block, wu)):
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            want = call(x, v)
            with torch.no_grad():
                assert torch.equal(call(leaf(x), leaf(v)), want)
            with torch.inference_mode():
                assert torch.equal(call(x, v), want)
        for args in ((leaf(x), v), (x, leaf(v)), (leaf(x) * 1, leaf(v))):
            with pytest.warns(UserWarning, match="autograd") as caught:
                y = call(*args)
            assert torch.equal(y, want) and not y.requires_grad
            assert caught[0].filename == __file__
        with torch.autograd.forward_ad.dual_level():
            with pytest.warns(UserWarning, match="autograd"):
                call(torch.autograd.forward_ad.make_dual(x, x), v)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with pytest.raises(UserWarning):                        # a warning made an error is raised as that
                call(leaf(x), v)
    # the gradients' calls are what a training step makes instead, with its parameters as they are
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            y, mean, rstd = sds.layer_norm(leaf(x), leaf(w), stats=True)
            _, kept = sds.gated_ffn(leaf(x), leaf(wg), wu, wd, keep=True)
        sds.layer_norm_backward(dy, leaf(x), leaf(w), mean, rstd)
        sds.gated_ffn_backward(dy, leaf(x), leaf(wg), wu, wd, kept)
