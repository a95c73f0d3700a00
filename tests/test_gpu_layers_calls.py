"""How the layer operators are called, on the GPU: reports of waits that gave up, errors, warnings, host threads."""

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


def test_first_calls_from_several_host_threads():
    """Four host threads make a process's first calls at once, through the C entries (which do not hold the interpreter's lock) and
    through the functions on tensors, each on a stream and with workspaces of its own: what they give alone, bit for bit."""
    import os
    import subprocess
    import sys
    code = """
import ctypes as C, threading, torch
import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb
lib = sds.load()
g = torch.Generator(device="cuda"); g.manual_seed(3)
rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
SIZES = [(40, 256, 512), (700, 512, 256), (9, 1000, 264), (2000, 136, 520)]
data = [(rnd(r, d), rnd(f, d) * d ** -0.5, rnd(f, d) * d ** -0.5, rnd(d, f) * f ** -0.5, rnd(r, d)) for r, d, f in SIZES]
torch.cuda.synchronize()


def raw(k, stream):
    x, wg, wu, wd, dy = data[k]
    (r, d), f, p = x.shape, wg.shape[0], (lambda t: t.data_ptr())
    s, n = sds.gated_ffn_bytes(r, d, f), C.c_size_t(0)
    assert lib.sds_layer_norm_workspace_bytes(r, d, C.byref(n)) == 0
    byte = lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")
    y, h, dx, dn = (torch.empty_like(x) for _ in range(4))
    gw, gu, gd, dw, db = (torch.empty_like(t) for t in (wg, wu, wd, x[0].float(), x[0].float()))
    m, q = (torch.empty(r, device="cuda") for _ in range(2))
    keep, ws, wb, wn, t = byte(s.keep_bytes), byte(s.forward_keep_bytes), byte(s.backward_bytes), byte(n.value), sb.SDS_BF16
    rc = [lib.sds_layer_norm(p(x), d, t, None, None, 0, r, d, 1e-5, p(y), d, t, p(m), p(q), stream),
          lib.sds_gated_ffn(p(y), d, t, r, d, f, p(wg), p(wu), p(wd), 0, p(h), d, p(keep), p(ws), ws.numel(), stream),
          lib.sds_gated_ffn_backward(p(dy), d, p(y), d, t, r, d, f, p(wg), p(wu), p(wd), p(keep), p(dn), d, p(gw), p(gu), p(gd), p(wb),
                                     wb.numel(), stream),
          lib.sds_layer_norm_backward(p(dn), d, t, p(x), d, t, None, 0, p(m), p(q), r, d, p(dx), d, p(dw), p(db), p(wn), wn.numel(), stream)]
    assert rc == [0] * 4, rc
    return [y, h, dn, gw, gu, gd, dx, dw, db], (keep, ws, wb, wn, m, q)


def tensors(k):
    x, wg, wu, wd, dy = data[k]
    y, m, q = sds.layer_norm(x, stats=True)
    h, keep = sds.gated_ffn(y, wg, wu, wd, keep=True)
    dn, gw, gu, gd = sds.gated_ffn_backward(dy, y, wg, wu, wd, keep)
    return [y, h, dn, gw, gu, gd, *sds.layer_norm_backward(dn, x, None, m, q)]


got, failed, gate = [[] for _ in SIZES], [], threading.Barrier(len(SIZES))


def work(k):
    try:
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            gate.wait(60)
            kept = []
            for _ in range(5):
                out, more = raw(k, stream.cuda_stream)
                kept.append(more)
                got[k] += [out, tensors(k)]
            stream.synchronize()
    except BaseException as e:
        failed.append(repr(e))


threads = [threading.Thread(target=work, args=(k,)) for k in range(len(SIZES))]
[t.start() for t in threads]
[t.join() for t in threads]
assert not failed, failed
torch.cuda.synchronize()
for k in range(len(SIZES)):
    want = tensors(k)
    torch.cuda.synchronize()
    assert len(got[k]) == 10
    for out in got[k]:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
sds.gated_ffn_status()
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=root, timeout=240)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout[-500:] + r.stderr[-2000:]


def test_rows_that_overlap_are_a_bad_argument():
    """Broadcast rows (a stride of zero, as the gradient of a sum has) and overlapping windows, as input, gradient or output: a
    ValueError that names the argument, on the host."""
    x, wg, wu, wd, dy = ffn_inputs(6, 64, 64, BF16, 43)
    _, mean, rstd = sds.layer_norm(x, stats=True)
    _, kept = sds.gated_ffn(x, wg, wu, wd, keep=True)
    row, windows = x[:1].expand(6, 64), torch.as_strided(x, (6, 64), (8, 1))
    for bad in (row, windows):
        for call in (lambda: sds.layer_norm(bad), lambda: sds.gated_ffn(bad, wg, wu, wd), lambda: sds.layer_norm(x, out=bad),
                     lambda: sds.gated_ffn(x, wg, wu, wd, out=bad), lambda: sds.layer_norm_backward(bad, x, None, mean, rstd),
                     lambda: sds.layer_norm_backward(dy, bad, None, mean, rstd), lambda: sds.gated_ffn_backward(bad, x, wg, wu, wd, kept),
                     lambda: sds.gated_ffn_backward(dy, bad, wg, wu, wd, kept)):
            with pytest.raises(ValueError, match="overlap"):
                call()
    one = x[:1].expand(1, 64)                                        # (a single row overlaps nothing)
    assert torch.equal(sds.layer_norm(one), sds.layer_norm(x)[:1])
    assert torch.equal(sds.layer_norm(row.contiguous())[5], sds.layer_norm(x)[0])
