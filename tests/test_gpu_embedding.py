"""Embedding lookup and its gradient by sorted tokens.  The lookup is exact (one product in fp32, one rounding).  A sum of the
gradient has at most 128 roundings within a chunk and 160 where chunks are joined: 2e-5 of the sum of magnitudes."""
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_layernorm import matrix
from test_gpu_logprobs import BF, F32

pytestmark = pytest.mark.gpu


def lookup(table, ids, out, scale=1.0, padding=-1, status=B.OK):
    ws = B.alloc_workspace(B.embedding_workspace_bytes())
    B.embedding_forward(table, ids, out, ws, scale=scale, padding_id=padding)
    assert B.last_device_status(ws) == status
    return out


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,V,d,pad,start", [(1, 1, 1, 0, 0), (5, 3, 8, 0, 0), (9, 100, 33, 1, 1), (300, 5000, 1024, 0, 0), (77, 1000, 1025, 3, 0),
                                             (2, 10, 20000, 0, 0), (70000, 50, 16, 0, 0)])
def test_lookup(n, V, d, pad, start, dtype):
    table = matrix(V, d, dtype, pad, start)
    ids = torch.randint(V, (n,), device="cuda")
    want = (table[ids].float() * 45.25).to(dtype)
    buf = torch.full((n + 2, d + 2 * pad + 8), 3.0, dtype=dtype, device="cuda")
    out = buf[1:n + 1, pad:pad + d] if pad else buf[1:n + 1, 8:8 + d]
    lookup(table, ids, out, 45.25)
    assert torch.equal(out, want)
    out.fill_(3.0)
    assert (buf == 3).all()
    ids[n // 2] = 0
    lookup(table, ids, out, 45.25, padding=0)
    assert torch.equal(out, torch.where((ids == 0)[:, None], 0.0, (table[ids].float() * 45.25)).to(dtype))


def test_ids_outside_the_table():
    table = matrix(10, 24, BF)
    ids = torch.tensor([1, 10, -1, 9, -7], device="cuda")
    out = lookup(table, ids, torch.empty(5, 24, dtype=BF, device="cuda"), padding=-1, status=B.E_BAD_LABEL)
    assert torch.equal(out[[0, 3]], table[[1, 9]]) and (out[[1, 2, 4]] == 0).all()
    lookup(table, torch.tensor([1, -1], device="cuda"), out[:2], padding=-1)


def gradient(dy, ids, V, scale=1.0, padding=-1, accumulate=False, start=7.0, status=B.OK, ws=None):
    n, d = dy.shape
    table = torch.full((V, d), start, device="cuda")
    ws = B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, d)) if ws is None else ws
    B.embedding_backward(dy, ids, table, ws, scale=scale, padding_id=padding, accumulate=accumulate)
    assert B.last_device_status(ws) == status
    return table


def check(dy, ids, V, scale=1.0, padding=-1):
    n, d = dy.shape
    part = (ids != padding) & (ids >= 0) & (ids < V)
    zero = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    src = torch.where(part[:, None], dy.double(), 0.0)
    at = torch.where(part, ids, 0)
    want, size = zero.index_add(0, at, src) * scale, zero.index_add(0, at, src.abs()) * abs(scale)
    got = gradient(dy, ids, V, scale, padding)
    assert ((got.double() - want).abs() <= 2e-5 * size).all()
    added = gradient(dy, ids, V, scale, padding, True, 0.5)
    assert ((added.double() - want - 0.5).abs() <= 2e-5 * size + 2.0 ** -23 * (want.abs() + 0.5)).all()
    assert torch.equal(gradient(dy, ids, V, scale, padding), got)
    named = torch.zeros(V, dtype=torch.bool, device="cuda")
    named[ids[part]] = True
    assert (added[~named] == 0.5).all() and (got[~named] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,V,d,pad,start", [
    (1, 1, 1, 0, 0), (2, 300, 8, 0, 0), (50, 4096, 256, 0, 0), (9, 100, 33, 1, 1), (1000, 255, 64, 0, 0), (1000, 256, 40, 5, 0), (5000, 65535, 16, 0, 0),
    (5000, 65536, 24, 0, 0), (20000, 152064, 128, 0, 0), (777, 1000, 2056, 0, 0), (3000, 17, 4099, 0, 1), (70001, 5000, 32, 0, 0)])
def test_gradient(n, V, d, pad, start, dtype):
    ids = torch.randint(V, (n,), device="cuda")
    check(matrix(n, d, dtype, pad, start), ids, V, 0.75)


@pytest.mark.parametrize("kind", ["one", "two", "half", "sorted", "reversed", "last", "steps"])
@pytest.mark.parametrize("n", [7, 100, 4097, 30000])
def test_gradient_of_crowds(kind, n):
    V, i = 20000, torch.arange(n, device="cuda")
    ids = {"one": torch.full_like(i, 123), "two": 5 + 1000 * (i % 2), "half": torch.where(i % 2 == 0, 77, (i * 7919) % V), "sorted": i % V,
           "reversed": (n - 1 - i) % V, "last": torch.full_like(i, V - 1), "steps": i // 13 % V}[kind]
    check(matrix(n, 64, BF), ids, V)
    check(matrix(n, 64, F32), ids, V, 2.0, int(ids[0]))       # its first token is padding


def test_gradient_of_ids_outside():
    dy = matrix(6, 16, F32)
    ids = torch.tensor([3, 20, -5, 3, 19, -1], device="cuda")
    got = gradient(dy, ids, 20, status=B.E_BAD_LABEL)
    assert torch.allclose(got[3], dy[0] + dy[3]) and torch.equal(got[19], dy[4]) and (got[[0, 1, 2] + list(range(4, 19))] == 0).all()
    assert (gradient(dy, torch.full((6,), -1, device="cuda"), 20) == 0).all()
    assert (gradient(dy, torch.full((6,), -1, device="cuda"), 20, accumulate=True) == 7).all()


def test_wide_key_range():
    """ids of four digits; the table's rows are not all there, so it is added to"""
    V, n = 30_000_000, 3000
    ids = torch.randint(V, (n,), device="cuda")
    ids[:100] = V - 1
    dy = matrix(n, 1, F32)
    table = torch.zeros(V, 1, device="cuda")
    ws = B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, 1))
    B.embedding_backward(dy, ids, table, ws, accumulate=True)
    want = torch.zeros(V, 1, dtype=torch.float64, device="cuda").index_add(0, ids, dy.double())
    assert ((table.double() - want).abs() <= 2e-5 * 100).all()


def test_lookup_of_many_tokens_with_ids_outside():
    """more than one block looks through"""
    n = 20000
    table, ids = matrix(100, 8, BF), torch.randint(100, (n,), device="cuda")
    out = lookup(table, ids, torch.empty(n, 8, dtype=BF, device="cuda"))
    assert torch.equal(out, table[ids])
    ids[n - 1] = 100
    out = lookup(table, ids, out, status=B.E_BAD_LABEL)
    assert torch.equal(out[:-1], table[ids[:-1]]) and (out[-1] == 0).all()
    ids[n - 1] = -1
    lookup(table, ids, out)
