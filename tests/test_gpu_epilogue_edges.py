"""Products with epilogue whose rows are aligned and whose columns end inside a 16-byte group: what lies between a row's last
column and the next row is left as it was."""
import pytest
import torch

from test_gpu_epilogue import check_forward, fence_ok, padded, rand
from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("N", [1, 5, 17, 23, 32 + 4, 95, 250, 257, 300, 509, 815])
@pytest.mark.parametrize("M", [100, 129, 300])
def test_columns_that_end_inside_a_group(M, N, residual, act):
    """All of C, residual and pre in rows of the next multiple of 8 columns, and of one more 8."""
    to = -N % 8 + (8 if N % 8 == 0 else 0)
    check_forward(M, N, 72, act, torch.bfloat16, residual=residual, pre=False, extra=to)
    A, W, b = rand(0, M, 72, dtype=torch.bfloat16), rand(1, N, 72, dtype=torch.bfloat16), rand(2, N, dtype=torch.bfloat16)
    R, rbuf = padded(rand(3, M, N, dtype=torch.bfloat16), to + 8) if residual else (None, None)
    (Y, ybuf), (Z, zbuf), (Y2, _), (Z2, _) = (padded(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), x) for x in (to, to + 8, 3, 5))
    B.gemm_epilogue(A, W, Y, bias=b, activation=act, residual=R, pre=Z)
    assert fence_ok(ybuf, N) and fence_ok(zbuf, N) and (R is None or fence_ok(rbuf, N))
    # Rows that start anywhere: the same sums, so the same z, and the same C where nothing but the residual is added to it.  The
    # product that ends GELU may be rounded before the residual is added in one kernel and not in the other, 2^-24 of it, and the
    # sums differ by that and a rounding of their own each, 2^-24 of the sum; rounded to bf16 once each, 2^-8 of it.
    B.gemm_epilogue(A, W, Y2, bias=b, activation=act, residual=R, pre=Z2)
    assert torch.equal(Z, Z2)
    if act == "none" or not residual:
        assert torch.equal(Y, Y2)
    else:
        y, f = Y.double(), Y.double() - R.double()
        assert bool(((y - Y2.double()).abs() <= 2.0 ** -24 * f.abs() + (2.0 ** -23 + 2.0 ** -7) * 1.01 * y.abs()).all())
    if residual:
        B.gemm_epilogue(A, W, R, bias=b, activation=act, residual=R)
        assert torch.equal(R, Y) and fence_ok(rbuf, N)


def test_neighbouring_outputs_in_one_buffer():
    """C and pre of two products side by side in the rows of one buffer."""
    M, K, widths = 400, 128, (300, 20, 4, 188)
    buf = torch.zeros(M, 512, dtype=torch.bfloat16, device="cuda")
    A = rand(0, M, K, dtype=torch.bfloat16)
    parts, want, at = [], [], 0
    for i, n in enumerate(widths):
        W = rand(1 + i, n, K, dtype=torch.bfloat16)
        parts.append((W, buf[:, at:at + n]))
        want.append(torch.empty(M, n, dtype=torch.bfloat16, device="cuda"))
        B.gemm_epilogue(A, W, want[-1], activation="silu")
        at += n
    for W, out in reversed(parts):
        B.gemm_epilogue(A, W, out, activation="silu")
    for (_, out), w in zip(parts, want):
        assert torch.equal(out, w)
