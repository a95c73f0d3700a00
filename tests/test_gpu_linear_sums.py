"""Sums of float results of the linear layer, of terms of one sign, in every form of the product.

The tensor cores truncate as they add 16 products to an accumulator: an addition loses less than a unit in the last place of the
running sum, 2 u = 2^-23 of it. With m additions of terms of one sign the running sum is j / m of the last one behind the j-th, so an
accumulator loses at most 2 u (1 + ... + m) / m = (m + 1) u of itself. At most 16 steps of K of 64 products, 64 additions, are left to one.
The accumulators' sums are then added in floats, rounded to nearest: up to 24 roundings of either sign, sqrt(24) u at most in the mean square.
(In one accumulator 28 steps of such terms lose 4.4e-6, 32 lose 5.1e-6 and 128 more than 2e-5; the bound is 4.2e-6.)
"""
import pytest
import torch

import paper_2501_05370_b200 as sds

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
FEW = [(1, 8192, 32768), (16, 28672, 8192), (16, 28672, 8195), (7, 65536, 1000), (32, 8192, 24576), (64, 8192, 24576), (64, 24576, 20480), (33, 24576, 20483),
       (64, 40960, 264), (128, 16384, 8192), (128, 65536, 512), (100, 12288, 2051), (200, 131072, 300), (10, 163840, 130)]
MANY = [(300, 8192, 512), (700, 8192, 519), (3000, 8192, 519), (3000, 8192, 520), (1500, 16384, 1024)]


@pytest.mark.parametrize("rows,k,n", FEW + MANY)
def test_sums_of_one_sign(rows, k, n):
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    x = torch.randn(rows, k, generator=g, device="cuda").abs().to(BF16)
    w = (torch.randn(n, k, generator=g, device="cuda").abs() * k ** -0.5).to(BF16)
    y = sds.linear(x, w, out_dtype=F32)
    off, size, x = 0.0, 0.0, x.double()
    for c in range(0, n, 2048):
        want = x @ w[c:c + 2048].double().T
        off += float((y[:, c:c + 2048].double() - want).pow(2).sum())
        size += float(want.pow(2).sum())
    assert (off / size) ** 0.5 <= 65 * U + 24 ** 0.5 * U
    sds.linear_status()
