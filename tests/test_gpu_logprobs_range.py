"""Log-probabilities and their gradient over the range of temperatures and of logits, against the definitions in 64 bits.

Tolerances as in test_gpu_logprobs.py.  The gradient is compared with the formula's at the lse and entropy that it is given:
log p = z / tau - lse then comes from fused operations, off by 2^-22 of itself, where 1 / tau is a power of two (elsewhere by
2^-48 of |z / tau| more, which the sizes here do not see); probabilities below 2^-126 count as 0 (1e-30 beside them)."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_logprobs import BF, F32, SUM, check, half_step, logits_of, score, tokens_of

pytestmark = pytest.mark.gpu
f32 = lambda x: float(torch.tensor(x, dtype=F32))
TAUS = [1.0, f32(0.05), f32(0.7), f32(7.3), 2.0 ** -20, 2.0 ** 20]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("rows,V,k", [(3, 40001, 20), (200, 5003, 5)])
def test_temperatures(rows, V, k, tau, dtype):
    """logits of the temperature's size, and of a size of their own"""
    t = tokens_of(rows, V, ignored=1)
    check((logits_of(rows, V, F32) * tau).to(dtype), t, k, tau)
    if tau > 0.01:
        check(logits_of(rows, V, dtype), t, k, tau)


def formula(z, t, tau, lse, entropy, gp, gl, gh):
    """gradients and the sizes of their terms"""
    lp = z.double() / tau - lse.double()[:, None]
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, 0.0)
    hot = torch.zeros_like(lp).scatter_(1, t[:, None], 1.0)
    gp, gl, gh, ent = (x.double()[:, None] for x in (gp, gl, gh, entropy))
    size = (gp.abs() * (hot + p) + gl.abs() * p + gh.abs() * (plp.abs() + p * ent)) / tau
    return (gp * (hot - p) + gl * p - gh * (plp + p * ent)) / tau, size


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tau", [1.0, 2.0 ** -20, 2.0 ** 20])
@pytest.mark.parametrize("height", [0.0, 300.0, 1e7, 1e11, 1e13, 1e30, -300.0, -1e11, -1e13, -1e30])
def test_gradients_of_rows_at_any_height(height, tau, dtype):
    """one token at `height` (of z / tau), others 20, 200, a tenth or twice of it below, or masked"""
    V, n = 3001, 4
    z = torch.full((n, V), -math.inf, device="cuda", dtype=torch.float64)
    top = torch.tensor([5, 3000, 17, 18], device="cuda")
    z.scatter_(1, top[:, None], height)
    for r, below in enumerate((20.0, 200.0, 0.1 * abs(height) + 1, 2 * abs(height) + 1)):
        z[r, 100:1000] = height - below
    z[2, 200:300] = torch.finfo(F32).min / 2 / max(tau, 1.0)          # a mask of about the lowest value
    z = (z * tau).to(F32).to(dtype)
    one = torch.ones(n, device="cuda")
    fw = score(z, top, 0, tau)
    d = torch.full_like(z, 7.0)
    B.token_logprobs_backward(z, top, fw["lse"], fw["entropy"], d, d_logp=one, d_lse=0.5 * one, d_entropy=-0.25 * one, temperature=tau)
    want, size = formula(z, top, tau, fw["lse"], fw["entropy"], one, 0.5 * one, -0.25 * one)
    off = 3 * SUM + 2.0 ** -22 * (z.double() / tau - fw["lse"].double()[:, None]).abs()
    some = size > 0                                          # (|log p| < 746 there)
    assert ((d.double() - want).abs() <= (half_step(dtype) + off) * size + 1e-30 / tau)[some].all()
    assert (d[~some] == 0).all()
    assert (d[z == -math.inf] == 0).all() and torch.isfinite(d).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tau", TAUS)
def test_gradients_at_every_temperature(tau, dtype):
    rows, V = 6, 5003
    z, t = (logits_of(rows, V, F32) * tau).to(dtype), tokens_of(rows, V)
    z[1, 50:] = -math.inf
    t[1] = 3
    g = torch.Generator(device="cuda").manual_seed(5)
    gp, gl, gh = (torch.randn(rows, generator=g, device="cuda") for _ in range(3))
    fw = score(z, t, 0, tau)
    d = torch.full_like(z, 7.0)
    B.token_logprobs_backward(z, t, fw["lse"], fw["entropy"], d, d_logp=gp, d_lse=gl, d_entropy=gh, temperature=tau)
    want, size = formula(z, t, tau, fw["lse"], fw["entropy"], gp, gl, gh)
    assert ((d.double() - want).abs() <= (half_step(dtype) + 3 * SUM) * size + 1e-30 / tau).all()
