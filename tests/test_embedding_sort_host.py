"""The limit on the clusters of the embedding gradient's sort (host side)."""
from paper_2506_03077_b200 import binding as B
from paper_2506_03077_b200 import build as build_mod

P = 0x10000     # an aligned address that is never read: every call here is refused on the host


def test_the_limit_and_what_it_refuses():
    build_mod.build()
    lib = B.lib()
    cap = lib.streambp_test_sort_cluster
    assert cap(-1) == B.E_SHAPE and cap(17) == B.E_SHAPE
    try:
        assert cap(4) == 16
        need = lib.streambp_embedding_backward_workspace_bytes(65536, 100, 64)
        assert lib.streambp_embedding_backward(P, 64, P, 65536, 100, 64, 1, 1.0, -1, 0, P, P, need, None) == B.E_CUDA
        assert lib.streambp_last_launch_count() == 0
    finally:
        assert cap(16) == 4
    assert cap(16) == 16
