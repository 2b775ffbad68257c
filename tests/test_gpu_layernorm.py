"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances.  The mean is a sum of at most 100 roundings in a row (a thread's values, the warp, the warps), 100 2^-24 = 6e-6 of
the mean magnitude; the deviations carry it, the variance 6e-6 of itself more.  The backward takes mean and rstd as given:
its two row sums are good to 6e-6 of their magnitudes, its column sums (a block's rows, the joined blocks; at most 150
roundings) to 1e-5 of theirs.  Results are rounded once."""
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_logprobs import BF, F32, half_step

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(1, 1), (3, 2), (2, 8), (7, 33), (5, 256), (9, 257), (33, 1000), (4, 1024), (65, 1032), (3, 2048), (2, 4096), (700, 512), (6, 4100),
          (3, 8192), (2, 8191), (3, 8200), (2, 20001), (2000, 96)]


def matrix(n, d, dtype, pad=0, start=0, seed=0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = (torch.randn(n * (d + pad) + start + 8, generator=g, device="cuda") + mean).to(dtype)
    return buf[start:start + n * (d + pad)].view(n, d + pad)[:, :d]


def forward(x, gain, bias, y=None, eps=EPS):
    n = x.shape[0]
    y = torch.full_like(x, 7.0) if y is None else y
    mean, rstd = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    B.layernorm_forward(x, gain, bias, eps, y, mean, rstd)
    return y, mean, rstd


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("pad,start,offset", [(0, 0, 0.0), (8, 0, 30.0), (3, 1, 0.5)])
def test_forward(n, d, pad, start, offset, dtype):
    x = matrix(n, d, dtype, pad, start, mean=offset)
    gain, bias = matrix(1, d, dtype, seed=1, mean=1.0)[0].contiguous(), matrix(1, d, dtype, seed=2)[0].contiguous()
    y, mean, rstd = forward(x, gain, bias)
    f = x.double()
    var, mu = torch.var_mean(f, 1, unbiased=False)
    r = torch.rsqrt(var + EPS)
    size = f.abs().mean(1)
    assert ((mean.double() - mu).abs() <= 6e-6 * size + 2.0 ** -24 * mu.abs()).all()
    # the variance about a mean that is off by e is larger by e^2
    e = 6e-6 * size + 2.0 ** -24 * mu.abs()
    assert ((rstd.double() - r).abs() <= r * (1e-5 + 0.5 * e * e * r * r)).all()
    h = (f - mu[:, None]) * r[:, None]
    want = h * gain.double() + bias.double()
    bound = (2e-5 * h.abs() + ((1 + h.abs()) * e[:, None] * r[:, None])) * gain.double().abs() + (half_step(dtype) + 2.0 ** -22) * want.abs() \
        + 2.0 ** -22 * bias.double().abs() + 1e-30
    assert ((y.double() - want).abs() <= bound).all()
    # in place, and without what is optional
    assert torch.equal(forward(x, gain, bias, y=x)[0], y)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_forward_without_options(dtype):
    x = matrix(5, 640, dtype)
    one, zero = torch.ones(640, device="cuda", dtype=dtype), torch.zeros(640, device="cuda", dtype=dtype)
    full = forward(x, one, zero)[0]
    y = torch.empty_like(x)
    B.layernorm_forward(x, None, None, EPS, y)
    assert torch.equal(y, full)


def gradients(x, dy, gain, mean, rstd, add=None, dx="new", sums=True, accumulate=False, start=0.0):
    n, d = x.shape
    dx = torch.full_like(x, 7.0) if isinstance(dx, str) else dx
    dg, db = (torch.full((d,), start, device="cuda") for _ in range(2)) if sums else (None, None)
    ws = B.alloc_workspace(B.layernorm_workspace_bytes(n, d)) if sums else None
    B.layernorm_backward(dy, x, gain, mean, rstd, dx=dx, d_gain=dg, d_bias=db, add=add, workspace=ws, accumulate=accumulate)
    assert ws is None or B.last_device_status(ws) == B.OK
    return dx, dg, db


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("pad,start,with_add", [(0, 0, False), (8, 0, True), (3, 1, True)])
def test_backward(n, d, pad, start, with_add, dtype):
    x, dy = matrix(n, d, dtype, pad, start, mean=0.5), matrix(n, d, dtype, pad, start, seed=1)
    add = matrix(n, d, dtype, pad, start, seed=2) if with_add else None
    gain = matrix(1, d, dtype, seed=3, mean=1.0)[0].contiguous()
    _, mean, rstd = forward(x, gain, None)
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy.double() * gain.double()
    a, b = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    r = rstd.double()[:, None]
    want = (g - a - h * b) * r + (0 if add is None else add.double())
    size = (g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)) * r
    dx, dg, db = gradients(x, dy, gain, mean, rstd, add)
    assert ((dx.double() - want).abs() <= 2e-5 * size + (half_step(dtype) + 2.0 ** -22) * want.abs() + 1e-30).all()
    sums = ((dg, (dy.double() * h).sum(0), (dy.double() * h).abs().sum(0)), (db, dy.double().sum(0), dy.double().abs().sum(0)))
    for got, ref, s in sums:
        assert ((got.double() - ref).abs() <= 1e-5 * s + 1e-30).all()
    # added to what is there; each output alone; in place of each input
    _, dg2, db2 = gradients(x, dy, gain, mean, rstd, add, None, True, True, 0.5)
    for got, (_, ref, s) in zip((dg2, db2), sums):
        assert ((got.double() - ref - 0.5).abs() <= 1e-5 * s + 2.0 ** -23 * (ref.abs() + 0.5)).all()
    assert torch.equal(gradients(x, dy, gain, mean, rstd, add, sums=False)[0], dx)
    for which in range(3 if with_add else 2):
        # copies with the rows' layout (another alignment takes another order of the sums)
        args = [matrix(n, d, dtype, pad, start, seed=1), matrix(n, d, dtype, pad, start, mean=0.5), None]
        args[2] = matrix(n, d, dtype, pad, start, seed=2) if with_add else None
        got = gradients(args[1], args[0], gain, mean, rstd, args[2], args[which])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dg) and torch.equal(got[2], db)


def test_against_autograd_and_differences():
    x, dy = matrix(4, 37, F32).contiguous(), matrix(4, 37, F32, seed=1).contiguous()
    gain, bias = matrix(1, 37, F32, seed=2, mean=1.0)[0].contiguous(), matrix(1, 37, F32, seed=3)[0].contiguous()
    _, mean, rstd = forward(x, gain, bias)
    dx, dg, db = gradients(x, dy, gain, mean, rstd)
    X, G, C = (t.double().requires_grad_() for t in (x, gain, bias))
    y = torch.nn.functional.layer_norm(X, (37,), G, C, EPS)
    for got, want in zip((dx, dg, db), torch.autograd.grad(y, (X, G, C), dy.double())):
        assert ((got.double() - want).abs() <= 2e-5 * (1 + want.abs())).all()
    f = lambda v: (torch.nn.functional.layer_norm(v, (37,), gain.double(), bias.double(), EPS) * dy.double()).sum(1)
    h = 2.0 ** -8
    for j in (0, 36):
        up, down = x.double(), x.double()
        up[:, j] += h
        down[:, j] -= h
        assert ((dx[:, j].double() - (f(up) - f(down)) / (2 * h)).abs() <= 2e-4).all()


def test_constant_rows_and_nan_stay_in_their_row():
    x = matrix(4, 600, BF).contiguous()
    x[1] = 2.5
    x[2, 7] = float("nan")
    one = torch.ones(600, device="cuda", dtype=BF)
    y, mean, rstd = forward(x, one, None)
    assert (y[1] == 0).all() and mean[1] == 2.5 and torch.isnan(y[2]).all() and torch.isfinite(y[[0, 3]]).all()
