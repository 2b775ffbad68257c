"""Activations and their slopes over the whole range of the types: finite everywhere, and the limits 0, z and 1."""
import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_epilogue import ACTS, HALF, act64, f64, slope64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.filterwarnings("ignore:overflow")
def test_huge_arguments(act, dtype):
    big = [1e5, 1e10, 1e13, 1e17, 1.8e19, 1.9e19, 1e25, 3e38]
    z = torch.tensor([-x for x in big] + big, device="cuda").to(dtype)
    n = z.numel()
    W = torch.zeros(n, 16, device="cuda", dtype=dtype)
    W[:, 0] = z
    A = torch.zeros(1, 16, device="cuda", dtype=dtype)
    A[0, 0] = 1
    Y, dz = (torch.zeros(1, n, device="cuda", dtype=dtype) for _ in range(2))
    B.gemm_epilogue(A, W, Y, activation=act)
    ref = act64(f64(z)[None], act)
    assert np.isfinite(f64(Y)).all()
    assert (np.abs(f64(Y) - ref) <= (2.0 ** -19 + HALF[dtype]) * np.abs(ref)).all()
    B.gemm_epilogue_backward(torch.ones_like(Y), z[None].contiguous(), act, dz)
    assert np.array_equal(f64(dz), slope64(f64(z)[None], act))           # 0 and 1 are exact in every type
    # rows long enough for the aligned kernel, and one that starts anywhere
    for width in (64, 63):
        zz = z.repeat(8)[:width][None].contiguous()
        out = torch.empty_like(zz)
        B.gemm_epilogue_backward(torch.ones_like(zz), zz, act, out)
        assert np.array_equal(f64(out), slope64(f64(zz), act))
