"""Tensor-core products into fp32 whose rows are aligned and whose columns end inside a 16-byte group: what lies between a
row's last column and the next row is left as it was."""
import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu

FENCE = 7.0


def operand(gen, rows, cols):
    """[rows, cols] in bf16, rows on 16-byte boundaries, with NaN behind every row."""
    buf = torch.full((rows, cols + 8 + -cols % 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :cols] = torch.randn(rows, cols, generator=gen, device="cuda")
    return buf[:, :cols]


@pytest.mark.parametrize("op", [B.OP_NT, B.OP_NN, B.OP_TN])
@pytest.mark.parametrize("M,N,K", [(3, 65, 60), (100, 70, 200), (300, 1, 64), (300, 257, 77), (300, 1002, 64), (129, 287, 130), (260, 255, 8),
                                   (300, 260, 77)])
def test_columns_that_end_inside_a_group(op, M, N, K):
    gen = torch.Generator(device="cuda").manual_seed(M + N + K + op)
    A = operand(gen, *((K, M) if op == B.OP_TN else (M, K)))
    W = operand(gen, *((N, K) if op == B.OP_NT else (K, N)))
    a, w = A.double(), W.double()
    a, w = a.T if op == B.OP_TN else a, w.T if op == B.OP_NT else w
    ref, err = a @ w, K * 2.0 ** -24 * (a.abs() @ w.abs())              # fp32 sums of exact products in any order
    ld = N + 4 + -N % 4
    buf = torch.full((M + 1, ld), FENCE, device="cuda")
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside[:M, :N] = False
    C = buf[:M, :N]
    B.gemm(op, A, W, C, engine=2)
    assert bool(((C.double() - ref).abs() <= err).all()) and bool((buf[outside] == FENCE).all())
    B.gemm(op, A, W, C, accumulate=True, engine=2)
    assert bool(((C.double() - 2 * ref).abs() <= 2 * err + 2.0 ** -23 * ref.abs()).all()) and bool((buf[outside] == FENCE).all())
    # two segments and a neighbour in the same rows, one launch
    both = torch.full((M + 1, 2 * ld), FENCE, device="cuda")
    left, right = both[:M, :N], both[:M, ld:ld + N]
    B.gemm_grouped([(op, [(A, W), (A, W)], left, False), (op, [(A, W)], right, False)])
    assert bool(((left.double() - 2 * ref).abs() <= 4 * err).all()) and bool(((right.double() - ref).abs() <= err).all())
    rest = torch.ones_like(both, dtype=torch.bool)
    rest[:M, :N], rest[:M, ld:ld + N] = False, False
    assert bool((both[rest] == FENCE).all())
