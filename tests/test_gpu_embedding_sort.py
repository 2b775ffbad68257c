"""The embedding gradient's sort in the clusters that a device without room for larger ones has."""
import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_embedding import check, gradient
from test_gpu_layernorm import matrix
from test_gpu_logprobs import BF

pytestmark = pytest.mark.gpu


@pytest.fixture
def cap():
    f = B.lib().streambp_test_sort_cluster
    yield f
    f(16)


@pytest.mark.parametrize("n,V,d", [(129, 300, 16), (1025, 5, 8), (8192, 100000, 8), (8193, 600, 24), (32768, 152064, 16), (50001, 511, 8), (65535, 70000, 8),
                                   (65536, 512, 8)])
def test_clusters_of_eight(n, V, d, cap):
    """up to eight tokens a thread; a stable sort has one result, and so have the sums behind it"""
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(V, (n,), generator=g, device="cuda")
    dy = matrix(n, d, BF)
    want = gradient(dy, ids, V)
    assert cap(8) == 16
    check(dy, ids, V)
    assert torch.equal(gradient(dy, ids, V), want)
    cap(15)                                         # (no cluster of fifteen: eight)
    assert torch.equal(gradient(dy, ids, V), want)


def test_smaller_clusters_are_refused(cap):
    n, V, d = 65536, 1000, 8
    ids, dy = torch.zeros(n, dtype=torch.int64, device="cuda"), matrix(n, d, BF)
    ws, out = B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, d)), torch.full((V, d), 7.0, device="cuda")
    for blocks in (0, 1, 4, 7):
        cap(blocks)
        assert B.embedding_backward(dy, ids, out, ws, check=False) == B.E_CUDA
    assert (out == 7).all()
    cap(8)
    B.embedding_backward(dy[:100], ids[:100], out, ws)
    assert B.last_device_status(ws) == B.OK
