"""Calls of the linear layer through the C entries, as a program without torch makes them: arrays inside larger buffers.

Tolerances as in test_gpu_linear.py: what is compared here has the same bits wherever it lies.
"""
import ctypes as C

import pytest
import torch

import paper_2501_05370_b200 as sds
from paper_2501_05370_b200 import binding as sb

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: sb.SDS_F32, BF16: sb.SDS_BF16, F16: sb.SDS_F16}


def randn(seed, *s):
    return torch.randn(*s, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


class Buffer:
    """[rows, n] at `shift` elements behind an allocation's begin, with a border that has to stay as it was."""

    def __init__(self, rows, n, t, shift):
        self.all = torch.full((rows * n + 64,), 7.0, device="cuda", dtype=t)
        self.inside = self.all[shift:shift + rows * n].view(rows, n)
        self.shift, self.count = shift, rows * n

    def ptr(self):
        return self.inside.data_ptr()

    def border_is_whole(self):
        return bool((self.all[:self.shift] == 7).all() and (self.all[self.shift + self.count:] == 7).all())


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("rows,n,steps", [(40, 24, 5), (700, 256, 6), (700, 264, 250), (5000, 72, 3), (300, 131, 9)])
@pytest.mark.parametrize("shift", [0, 1, 4, 8])
def test_gradient_of_a_table_anywhere_in_a_buffer(rows, n, steps, shift, t):
    """dtable lies at 0, 2, 8 and 16 bytes from a 16-byte boundary, db at 0, 4, 16 and 32: the same bits, and nothing beside them."""
    k = 64
    x, w, b = randn(1, rows, k).to(t), (0.1 * randn(2, n, k)).to(t), randn(3, n)
    table, dy = randn(4, steps, n).to(t), randn(5, rows, n).to(t)
    step = torch.randint(0, steps, (rows,), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda", dtype=torch.int32)
    kept = sds.linear(x, w, b, "silu", table=table, step=step, keep=True)[1]
    want = sds.linear_backward(dy, x, w, kept, bias=b, table=table, step=step)
    layer = sb.SdsLinearLayer(k, n, steps, CODE[t], sb.SDS_ACT_SILU, w.data_ptr(), b.data_ptr(), sb.SDS_F32, table.data_ptr())
    sizes = sb.SdsLinearSizes()
    assert sb.load().sds_linear_bytes(C.byref(layer), rows, C.byref(sizes)) == sb.SDS_OK
    ws = torch.empty(sizes.backward_bytes, device="cuda", dtype=torch.uint8)
    dtable, db = Buffer(steps, n, t, shift), Buffer(1, n, F32, shift)
    rc = sb.load().sds_linear_backward(C.byref(layer), dy.data_ptr(), n, CODE[t], x.data_ptr(), k, step.data_ptr(), rows, kept.data_ptr(), None, k, None,
                                       db.ptr(), dtable.ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == sb.SDS_OK
    assert torch.equal(dtable.inside, want[3]) and torch.equal(db.inside[0], want[2])
    assert dtable.border_is_whole() and db.border_is_whole()
