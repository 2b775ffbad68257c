"""The layer norm's gradient where the rows under way reuse their places in shared memory, on both sides of the widths at which
another kernel takes over, and without a gain; against the formulas in 64 bits.

Tolerances: as in test_gpu_layernorm.py (row sums to 6e-6 of their magnitudes, one rounding of dx), but that a block walks more
rows here: its column sums have as many roundings as it has rows (of 148 blocks or more), the joined sums at most 80 (up to
1184 blocks in 32 sections, the sections, a block's four warps), and each product 2, every one 2^-24 of the sum of magnitudes."""
import pytest
import torch

from test_gpu_layernorm import forward, gradients, matrix
from test_gpu_logprobs import BF, F32, half_step

pytestmark = pytest.mark.gpu


def compare(n, d, dtype, with_gain, with_add, pad=0, start=0):
    x, dy = matrix(n, d, dtype, pad, start, mean=0.5), matrix(n, d, dtype, pad, start, seed=1)
    add = matrix(n, d, dtype, pad, start, seed=2) if with_add else None
    gain = matrix(1, d, dtype, seed=3, mean=1.0)[0].contiguous() if with_gain else None
    _, mean, rstd = forward(x, None, None)
    dx, dg, db = gradients(x, dy, gain, mean, rstd, add)
    sums = torch.zeros(4, d, device="cuda", dtype=torch.float64)
    for r in range(0, n, 4096):         # (a part of the rows at a time)
        s = slice(r, r + 4096)
        rs = rstd[s].double()[:, None]
        h = (x[s].double() - mean[s].double()[:, None]) * rs
        g = dy[s].double() * (gain.double() if with_gain else 1.0)
        want = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * rs + (add[s].double() if with_add else 0.0)
        size = (g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)) * rs
        assert ((dx[s].double() - want).abs() <= 2e-5 * size + (half_step(dtype) + 2.0 ** -22) * want.abs() + 1e-30).all()
        dyh = dy[s].double() * h
        sums += torch.stack((dyh.sum(0), dyh.abs().sum(0), dy[s].double().sum(0), dy[s].double().abs().sum(0)))
    off = (n / min(n, 148) + 80 + 2) * 2.0 ** -24
    assert ((dg.double() - sums[0]).abs() <= off * sums[1]).all() and ((db.double() - sums[2]).abs() <= off * sums[3]).all()
    # dx alone, the sums alone, and all in the place of x
    assert torch.equal(gradients(x, dy, gain, mean, rstd, add, sums=False)[0], dx)
    assert torch.equal(gradients(x, dy, gain, mean, rstd, add, None)[1], dg)
    again = gradients(x, dy, gain, mean, rstd, add, x)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dg) and torch.equal(again[2], db)


@pytest.mark.parametrize("with_gain,with_add", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("n,d,dtype", [
    (16384, 4096, BF), (9001, 4096, BF), (5000, 8192, BF), (4001, 4104, BF), (20000, 1024, BF), (3500, 2048, F32), (2000, 8192, F32),
    (30001, 768, BF), (40000, 512, BF), (50000, 256, BF), (65536, 64, BF), (30000, 384, F32), (40001, 512, F32),
    (2100, 16384, BF), (1500, 12288, F32), (1501, 8200, BF)])
def test_places_used_again(n, d, dtype, with_gain, with_add):
    """so many rows that every ring's places are filled several times"""
    compare(n, d, dtype, with_gain, with_add)


@pytest.mark.parametrize("with_gain", [True, False])
@pytest.mark.parametrize("n,d,dtype,with_add", [
    (1000, 8872, F32, True), (1000, 8876, F32, True), (700, 13312, F32, False), (700, 13316, F32, False), (700, 16384, BF, True), (700, 16392, BF, True),
    (700, 17744, BF, True), (1000, 8192, F32, True), (1000, 8196, F32, True), (1000, 8192, BF, True), (1000, 8200, BF, False)])
def test_widths_beside_another_kernels(n, d, dtype, with_add, with_gain):
    """208 KB hold two rows of three (two) streams: 8872 (13312) fp32 columns; 16384 columns are a block's; 8192 are held in registers"""
    compare(n, d, dtype, with_gain, with_add)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d,pad,start", [(3, 1, 0, 0), (7, 33, 0, 0), (600, 1537, 3, 1), (2000, 4097, 0, 0), (5, 8191, 1, 0), (9, 8200, 3, 1), (3, 20001, 0, 0),
                                           (2, 32768, 0, 0), (4, 64, 8, 0), (100, 4096, 8, 0)])
@pytest.mark.parametrize("with_add", [False, True])
def test_gradients_without_a_gain(n, d, pad, start, with_add, dtype):
    compare(n, d, dtype, False, with_add, pad, start)
    # and of a gain of ones: the same products
    x, dy = matrix(n, d, dtype, pad, start, mean=0.5), matrix(n, d, dtype, pad, start, seed=1)
    _, mean, rstd = forward(x, None, None)
    one = torch.ones(d, device="cuda", dtype=dtype)
    for a, b in zip(gradients(x, dy, None, mean, rstd), gradients(x, dy, one, mean, rstd)):
        assert torch.equal(a, b)


