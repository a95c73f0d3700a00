"""The gated denoiser (residual blocks of layer norm and gated feed-forward, the layer operators inside the sampler)
against the oracle, which rounds to bfloat16 at the same points. Rows agree within 2e-2 relative, as the other bf16
denoisers' do."""
import numpy as np
import pytest

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb
from oracle import sds_oracle as o
import workloads as wl
from helpers import BAND, assert_rows_close, ell_close

pytestmark = pytest.mark.gpu

TOL = 2e-2


def _workload(d, f, nblock, K, B, L, activation="silu"):
    return wl.WORKLOADS["cfg3"].scaled(d=d, B=B, L=L, K=K, denoiser="gated", gated=dict(f=f, nblock=nblock, activation=activation))


def _oracle(gp):
    f64 = lambda v: [wl.bf16_bits_to_f32(x).astype(np.float64) if x is not None else None for x in v]
    wg, wu, wd, te = f64(gp.w_gate), f64(gp.w_up), f64(gp.w_down), f64(gp.temb)
    return lambda x, k: o.gated_forward(x, k, wg, wu, wd, gp.norm_w, gp.norm_b, te, gp.activation)


@pytest.mark.parametrize("d,f,nblock,rows,activation", [(128, 256, 1, 300, "silu"), (72, 200, 3, 77, "gelu"),
                                                        (256, 512, 2, 1000, "gelu_tanh"), (1000, 264, 2, 129, "silu"),
                                                        (64, 64, 4, 5, "silu"), (2048, 512, 1, 2500, "silu")])
def test_rows(d, f, nblock, rows, activation):
    import torch
    K = 9
    w = _workload(d, f, nblock, K, rows, 1, activation)
    gp = w.gated_params()
    if nblock > 1:
        gp.temb[1] = None                                            # a block without an embedding, one without a norm weight
        gp.norm_w[nblock - 1] = gp.norm_b[nblock - 1] = None
    s = sds.sampler_for(w, gated=gp)
    den = _oracle(gp)
    rng = np.random.default_rng(5)
    x = rng.standard_normal((rows, d)).astype(np.float32)
    k = rng.integers(0, K, size=rows).astype(np.int32)
    xt, kt = torch.from_numpy(x).cuda(), torch.from_numpy(k).cuda()
    out = s.denoise(xt, kt).cpu().numpy()
    assert np.array_equal(x, xt.cpu().numpy())                       # the input rows stay
    for r in list(range(0, rows, max(1, rows // 40))) + [rows - 1]:
        assert_rows_close(out[r], den(x[r].astype(np.float64), int(k[r])), TOL, r)
    # any number of rows: the same bits (1 row, and halves of the batch, alone)
    for n in sorted({1, rows // 2}):
        part = s.denoise(xt[:n].contiguous(), kt[:n].contiguous()).cpu().numpy()
        assert np.array_equal(part, out[:n])
    s.close()


def test_windows_replayed_and_free_run():
    """Every position of some windows: accept tests and reflections from the GPU's own outputs, outputs against the oracle."""
    w = _workload(256, 384, 2, 40, 70, 8)
    gp = w.gated_params()
    s = sds.sampler_for(w, gated=gp, seed=31, chain_id_offset=7)
    den = _oracle(gp)
    a, c, sig, _ = sds.schedule_for(w)
    a, c, sig = (v.astype(np.float64) for v in (a, c, sig))
    s.set_option(s.OPT_VERIFY_EARLY_EXIT, 0)
    s.reset()
    band = tests = 0
    for _ in range(3):
        na = int(s.get(sb.GET_CTL)[0])
        act, rowoff, n, Dc = s.get(sb.GET_ACT)[:na], s.get(sb.GET_ROWOFF)[:na + 1], s.get(sb.GET_N), s.get(sb.GET_DC)
        s.draft()
        X, T = s.get(sb.GET_X), s.get(sb.GET_TAIL)
        s.verify_window()
        Dq, ell, logU, mask = s.get(sb.GET_DQ), s.get(sb.GET_ELL), s.get(sb.GET_LOGU), s.get(sb.GET_ACCMASK)
        for si, b in enumerate(act):
            nb = int(n[b])
            Lt, r0 = min(w.L, w.K - nb), int(rowoff[si])
            W = np.concatenate([X[r0:r0 + Lt], T[b:b + 1]]).astype(np.float64)
            if b % 10 == 0:
                for j in range(Lt):
                    assert_rows_close(Dq[r0 + j], den(W[j], nb + j), TOL, (int(b), j))
            v = o.verify_window(W, Dq[r0:r0 + Lt], Dc[b], a, c, sig, nb, logU[b, :Lt].astype(np.float64))
            for j in range(Lt):
                assert ell_close(float(ell[b, j]), float(v["ell"][j]))
                tests += 1
                if abs(float(v["ell"][j]) - float(logU[b, j])) < BAND:
                    band += 1
                else:
                    assert bool((int(mask[b]) >> j) & 1) == bool(v["acc"][j])
        s.advance()
    assert band <= max(2, 2e-3 * tests)
    s.set_option(s.OPT_VERIFY_EARLY_EXIT, 1)
    out, calls, rows = [v.cpu().numpy() for v in s.sample_all()]
    assert np.all(np.isfinite(out)) and np.array_equal(s.get(sb.GET_N), np.full(70, 40))
    again = s.sample_all()[0].cpu().numpy()
    assert np.array_equal(out, again)
    s.close()


def test_drafter_at_the_state_accepts_its_first_position():
    """Drafter evaluated at Y_n: the batched pass gives row 1 the same bits, so position 1 has Delta = 0 and always passes."""
    w = _workload(128, 256, 2, 24, 300, 6)
    w.drafter_mode = sb.SDS_FROZEN_EXACT
    s = sds.sampler_for(w, gated=w.gated_params())
    s.set_option(s.OPT_VERIFY_EARLY_EXIT, 0)
    s.reset()
    for _ in range(3):
        act = s.get(sb.GET_ACT)[:int(s.get(sb.GET_CTL)[0])]
        s.draft()
        s.verify_window()
        assert np.all(s.get(sb.GET_S1)[act, 0] == 0.0) and np.all(s.get(sb.GET_ACCMASK)[act] & 1)
        s.advance()
    s.close()


def test_gated_network_as_independent_drafter_and_staged_windows():
    w = _workload(128, 256, 2, 30, 40, 5)
    gp = w.gated_params()
    small = wl.gated_params(77, 128, 64, 1, 30)
    s = sds.sampler_for(w, gated=gp, drafter=sds.drafter_for(w, gated=small))
    out, calls, rows = [v.cpu().numpy() for v in s.sample_all()]
    assert np.all(np.isfinite(out)) and np.array_equal(s.get(sb.GET_N), np.full(40, 30))
    s.close()
    s = sds.sampler_for(w, gated=gp)
    whole = s.sample_all()[0].cpu().numpy()
    s.set_option(s.OPT_STAGED_WINDOWS, 2)
    assert np.array_equal(s.sample_all()[0].cpu().numpy(), whole)
    s.close()


def test_layer_calls_give_the_denoisers_rows():
    """The public layer operators, one after the other on the same weights, against the denoiser's output."""
    import torch
    w = _workload(256, 512, 2, 6, 400, 1)
    gp = w.gated_params()
    s = sds.sampler_for(w, gated=gp)
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.standard_normal((400, 256)).astype(np.float32)).cuda()
    k = torch.from_numpy(rng.integers(0, 6, size=400).astype(np.int32)).cuda()
    want = s.denoise(x, k)
    bf = lambda b: torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda().view(torch.bfloat16)
    r = x
    for l in range(2):
        r = r + bf(gp.temb[l]).float()[k.long()]
        n = sds.layer_norm(r, torch.from_numpy(gp.norm_w[l]).cuda(), torch.from_numpy(gp.norm_b[l]).cuda(), 1e-5, out_dtype=torch.bfloat16)
        r = r + sds.gated_ffn(n, bf(gp.w_gate[l]), bf(gp.w_up[l]), bf(gp.w_down[l])).float()
    # (the public call rounds the block's output to bfloat16 before it is added, half a step of it)
    assert float((r - want).norm() / want.norm()) <= 2.0 ** -8
    s.close()


def test_picard_drafter_and_misaligned_rows():
    import torch
    w = _workload(128, 256, 1, 20, 30, 4)
    s = sds.sampler_for(w, gated=w.gated_params(), picard=sds.picard_for(w, 2))
    out = s.sample_all()[0].cpu().numpy()
    assert np.all(np.isfinite(out)) and np.array_equal(s.get(sb.GET_N), np.full(30, 20))
    s.close()
    s = sds.sampler_for(w, gated=w.gated_params())
    buf = torch.zeros(4 * 128 + 1, device="cuda")
    k = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(sds.SdsError) as e:
        s.denoise(buf[1:].view(4, 128), k)
    assert e.value.code == sb.SDS_EUNSUPPORTED
    s.close()
