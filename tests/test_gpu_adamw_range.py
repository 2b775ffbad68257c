"""AdamW at the ends of the range of fp32: second moments below the smallest normal number."""
import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_adamw import E32

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
