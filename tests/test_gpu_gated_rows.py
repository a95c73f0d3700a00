"""The gated denoiser's norm over every width and many rows (its own form of the kernel: embedding added, stream kept), seen
through one block, against 64 bits.

Bound, element by element. r = x + temb is one rounding in float, the same in torch. The normed row is off by at most norm_bound
(test_gpu_layers.py) before it is rounded to bfloat16: where that interval holds a tie, the kernel's value may be the neighbour of the one
used here, `en` away. That moves G by at most dg = en |Wg|^T and U by du = en |Wu|^T, act(G) by at most (|act'(G)| + 2 dg) dg as |act''| < 2,
and h by dh = da (|U| + du) + |act(G)| du before its rounding, which adds half a step of dh. The rest is Ffn64's bound of the block's output
before its last rounding (here there is none), and two roundings in float, of r and of the sum with the stream. (At 16384
columns the bound is a tenth of the output's size; a weight in the wrong place changes n by a tenth of its spread and G, U with it.)
"""
import numpy as np
import pytest
import torch

import paper_2501_05370_b200 as sds
import workloads as wl
from test_gpu_layers import BF16, U, Ffn64, half, norm_bound, plain_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(40000, 64), (20000, 72), (20000, 256), (9001, 512), (9000, 1000), (5000, 2048), (2001, 4096), (1500, 8184), (700, 16384)])
def test_one_block_of_many_rows(rows, d):
    K = 7
    w = wl.WORKLOADS["cfg3"].scaled(d=d, B=rows, L=1, K=K, denoiser="gated", gated=dict(f=64, nblock=1, activation="silu"))
    gp = w.gated_params()
    s = sds.sampler_for(w, gated=gp)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    x = torch.randn(rows, d, generator=g, device="cuda")
    k = torch.randint(0, K, (rows,), generator=g, device="cuda", dtype=torch.int32)
    out = s.denoise(x, k).double()
    bits = lambda v: torch.from_numpy(np.ascontiguousarray(v).view(np.int16)).cuda().view(BF16)  # noqa: E731
    wg, wu, wd = bits(gp.w_gate[0]), bits(gp.w_up[0]), bits(gp.w_down[0])
    nw, nb = torch.from_numpy(gp.norm_w[0]).cuda(), torch.from_numpy(gp.norm_b[0]).cuda()
    r = x + bits(gp.temb[0]).float()[k.long()]
    n64, _, _, xhat = plain_norm(r, nw, nb, 1e-5)
    e = norm_bound(xhat, nw, nb, d)
    en = (n64 + e).to(BF16).double() - (n64 - e).to(BF16).double()
    ref = Ffn64(n64.to(BF16), wg, wu, wd, "silu", BF16)
    dg, du = en @ wg.double().abs().T, en @ wu.double().abs().T
    dh = (ref.da.abs() + 2 * dg) * dg * (ref.u.abs() + du) + ref.a.abs() * du
    lim = ref.ey + (1 + half(BF16)) * dh @ wd.double().abs().T + 2 * U * (r.double().abs() + out.abs())
    over = (out - r.double() - ref.y).abs() / lim
    assert float(over.max()) <= 1.0, (rows, d, float(over.max()), int(over.argmax()))
    s.close()
