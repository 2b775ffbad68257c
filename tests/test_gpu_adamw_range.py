"""AdamW at the ends of the range of fp32: second moments and divisors below the smallest normal number, roots at the ties
of the codes."""
import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_adamw import E32, mx8_values, plain_mx8

pytestmark = pytest.mark.gpu


def one_step(g, eps, lr=1.0, beta1=0.9, beta2=0.95, dtype=torch.float32):
    """The parameter (from 0) and the moments (from 0) after a first step."""
    t = {"param": torch.zeros_like(g, dtype=dtype), "grad": g, "m": torch.zeros_like(g), "v": torch.zeros_like(g)}
    B.adamw_step(B.AdamWPlan([t]), lr, beta1, beta2, eps, 1)
    return [t[k].double().cpu().numpy() for k in ("param", "m", "v")]


@pytest.mark.parametrize("eps", [0.0, 1e-20, 1e-22, 1e-8])
@pytest.mark.parametrize("n", [4096 * 3, 1001])
def test_second_moments_below_the_normal_range(eps, n):
    """Gradients from 1e-21 up: their second moments start among the subnormal numbers.  Held to the nearest multiple of
    2^-149, they are what the rest of the step is made of: the move is compared with the one that the stored moments give.
    Its bound: the root, its rate and their sum with eps are three roundings, the reciprocal's ulp two, the product with m,
    the rate and the last sum three."""
    g = torch.logspace(-21, -17, n, device="cuda") * torch.where(torch.arange(n, device="cuda") % 3 == 0, -1.0, 1.0)
    p, m, v = one_step(g, eps)
    g = g.double().cpu().numpy()
    assert (np.abs(m - 0.1 * g) <= 4 * E32 * np.abs(m)).all()
    # the products' own roundings, relative and of half a subnormal step each (the last after a factor of at most 1)
    assert (np.abs(v - 0.05 * g * g) <= 8 * E32 * v + 2.0 ** -149).all() and (v > 0).any() and (v[v > 0] < 2.0 ** -126).any()
    seen = v > 0                                  # where the square itself vanished, the formula has no more than eps to go by
    move = 10 * m[seen] / (np.sqrt(v[seen] / (1 - 0.95)) + eps)
    assert np.isfinite(p[seen]).all()
    assert (np.abs(p[seen] + move) <= 8 * E32 * np.abs(move)).all()


@pytest.mark.parametrize("state", ["f32", "mx8"])
@pytest.mark.parametrize("eps,lr,least,most", [(1e-39, 1e-17, -37, -24), (1e-40, 1e-17, -37, -24), (2.0 ** -130, 1e-17, -37, -24),
                                               (1e38, 1e37, -3, 0)])
def test_divisors_outside_the_normal_range(eps, lr, least, most, state):
    """eps alone is the divisor: beside a small one the squares of the gradients vanish in fp32, beside a huge one their roots
    do.  A parameter without a gradient stays, the others move by lr g / eps.  Bound: a small eps is the subnormal number
    that fp32 makes of it, so may m be for the smallest gradients (half a step of them); the constant and the product of m are two
    roundings, the reciprocal's ulp two, the product with m and the rate two; the parameter's own is one of the result."""
    n = 1024
    g = torch.logspace(least, most, n, device="cuda")
    g[::5] = 0
    t = {"param": torch.ones(n, device="cuda"), "grad": g}
    if state == "f32":
        t |= {k: torch.zeros(n, device="cuda") for k in ("m", "v")}
    else:
        t |= {k: torch.zeros(n, dtype=torch.uint8, device="cuda") for k in ("m", "v")}
        t |= {k: torch.ones(n // 32, dtype=torch.uint8, device="cuda") for k in ("m_scale", "v_scale")}
    B.adamw_step(B.AdamWPlan([t]), lr, 0.9, 0.95, eps, 1)
    p, x, eps = t["param"].double().cpu().numpy(), g.double().cpu().numpy(), float(np.float32(eps))
    move = lr * x / eps
    assert (p[x == 0] == 1).all() and move.max() > 1e-3
    assert (np.abs(p - (1 - move)) <= 6.01 * E32 * move + 10 * lr / eps * 2.0 ** -150 + E32 * np.abs(1 - move)).all()


def test_roots_at_the_ties_of_the_codes():
    """With beta2 = 0 the new second moment is x^2 rounded, and its root rounded to nearest is x again.  x lies halfway
    between two codes of its block, and a bit to either side, in every exponent that squares allow: a root that is off in its
    last bit leaves another code."""
    xs = []
    for e in range(-60, 61):
        for mant in range(8):
            tie = np.float32((1 + (mant + 0.5) / 8) * 2.0 ** e)
            xs += [np.nextafter(tie, np.float32(0)), tie, np.nextafter(tie, np.float32(np.inf)), np.float32(1.75 * 2.0 ** e)]
    n = len(xs)
    assert n % 32 == 0                            # one exponent to a block
    x = torch.from_numpy(np.array(xs, dtype=np.float32)).cuda()
    t = {"param": torch.zeros(n, device="cuda"), "grad": x, "weight_decay": 0.0}
    t |= {k: torch.zeros(n, dtype=torch.uint8, device="cuda") for k in ("m", "v")}
    t |= {k: torch.ones(n // 32, dtype=torch.uint8, device="cuda") for k in ("m_scale", "v_scale")}
    B.adamw_step(B.AdamWPlan([t]), 1e-3, 0.9, 0.0, 1e-8, 1)
    codes, scale = plain_mx8(x, keep=True)
    assert torch.equal(t["v"], codes) and torch.equal(t["v_scale"], scale)
    assert torch.equal(mx8_values(t["v"], t["v_scale"]), mx8_values(codes, scale))


def test_codes_under_the_smallest_scales():
    """Every code under scale bytes 1 .. 4: fp32 holds them all, bf16 those under 3 and more; finer ones are rounded to nearest."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(4)
    scales = torch.arange(1, 5, dtype=torch.uint8, device="cuda").repeat_interleave(8)
    ref = codes.view(torch.float8_e4m3fn).double() * torch.exp2(scales.double() - 127).repeat_interleave(32)
    some = ~torch.isnan(ref)
    out, rounded = torch.empty(1024, device="cuda"), torch.empty(1024, device="cuda", dtype=torch.bfloat16)
    B.mx8_decode(codes, scales, out)
    B.mx8_decode(codes, scales, rounded)
    assert torch.equal(out.double()[some], ref[some]) and bool(torch.isnan(out[~some]).all())
    # multiples of 2^-135 against bf16's of 2^-133, ties to even
    want = torch.where(ref.abs() < 2.0 ** -126, torch.round(ref * 2.0 ** 133) * 2.0 ** -133, ref)
    assert torch.equal(rounded.double()[some], want[some]) and bool(torch.isnan(rounded[~some]).all())
    exact = some & (torch.arange(1024, device="cuda") >= 512)
    assert torch.equal(rounded.double()[exact], ref[exact]) and not torch.equal(rounded.double()[some], ref[some])


@pytest.mark.parametrize("n", [1000, 200_000])
@pytest.mark.parametrize("most", [float("inf"), 3e38, 1.0])
def test_norms_that_overflow_fp32(n, most):
    """A finite sum of squares whose root is above fp32's range: the norm is infinite, the factor what the formula gives, 1 for
    no bound.  One launch and several."""
    t = {"param": torch.zeros(n, device="cuda"), "grad": torch.full((n,), 1e38, device="cuda")}
    t |= {k: torch.zeros(n, device="cuda") for k in ("m", "v")}
    plan, ws = B.AdamWPlan([t]), B.alloc_workspace(B.grad_norm_workspace_bytes())
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    B.grad_norm(plan, most, norm, scale, ws)
    want = min(1.0, float(np.float32(most)) / (float(np.float32(1e38)) * np.sqrt(float(n))))
    assert np.isinf(norm.item())
    # the result's rounding, of a subnormal number where the bound is small
    assert abs(scale.item() - want) <= E32 * want * 1.01 + 2.0 ** -150
    t["grad"].fill_(1e-3)
    B.grad_norm(plan, float("inf"), norm, scale, ws)
    assert scale.item() == 1.0


@pytest.mark.parametrize("eps,lr,size", [(1e-40, 1e-17, 1e-24), (1e-8, 1e-3, 1.0), (1e38, 1e37, 1.0)])
def test_step_number_on_the_device_under_any_eps(eps, lr, size):
    """The rates formed by the kernel from a step number in device memory and by the host, each from doubles rounded once: the
    moves differ by a rounding of each of the two rates at most."""
    g, out = torch.logspace(-3, 0, 999, device="cuda") * size, []
    for step in (3, torch.tensor([3], device="cuda")):
        t = {"param": torch.zeros_like(g), "grad": g, "m": torch.zeros_like(g), "v": torch.zeros_like(g)}
        B.adamw_step(B.AdamWPlan([t]), lr, 0.9, 0.95, eps, step)
        out.append(t["param"].double())
    assert bool((out[0] != 0).all()) and bool(((out[0] - out[1]).abs() <= 4 * E32 * out[0].abs()).all())
