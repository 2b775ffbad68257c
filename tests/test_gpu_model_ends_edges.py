"""Calls of a model's ends that the documentation allows and the other tests do not make: lists longer than what a mask leaves,
crowded rows, gains that start anywhere, one workspace for calls one after another, the workspaces' guards."""
import math
import os
import subprocess
import sys

import pytest
import torch

import test_gpu_layernorm as norms
from paper_2506_03077_b200 import binding as B
from test_gpu_distill import check as check_distill
from test_gpu_distill import teacher
from test_gpu_layernorm import EPS, forward, gradients, matrix
from test_gpu_logprobs import BF, F32, check, logits_of, reference, score

pytestmark = pytest.mark.gpu
GUARDED = "STREAMBP_WS_GUARD" in os.environ       # read by the library once per process: below, in one of its own


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,V", [(2, 33001), (200, 33000), (3, 1000), (160, 9)])
@pytest.mark.parametrize("left", [1, 5, 127])
@pytest.mark.parametrize("floor", [-math.inf, "lowest"])
def test_lists_longer_than_what_a_mask_leaves(rows, V, left, floor, dtype):
    z = logits_of(rows, V, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    keep = torch.zeros(rows, V, dtype=torch.bool, device="cuda").scatter_(1, torch.randint(V, (rows, left), generator=g, device="cuda"), True)
    z = torch.where(keep, z, torch.finfo(dtype).min if floor == "lowest" else floor)
    k = min(V, 128)
    got, ref = score(z, None, k), reference(z, None, k, 1.0)
    assert torch.equal(got["top_ids"], ref["top_ids"])
    assert (got["top_logp"].isneginf() == ref["top_logp"].isneginf()).all() and not got["entropy"].isnan().any()


@pytest.mark.parametrize("rows", [2, 160])
def test_many_large_values_in_few_threads(rows):
    """more values above the first bound than the candidates' list holds: every thousandth group, all of them different"""
    V = 400000
    i = torch.arange(V, device="cuda")
    z = torch.where((i // 4) % 1024 < 8, 50 + (i * 7919 % 100003) / 10000, -(i % 13).float()).expand(rows, V).contiguous()
    for k in (7, 24, 100):
        check(z, None, k)


def test_the_same_row_as_one_of_few_and_one_of_many():
    """blocks of either kind list and score alike"""
    z = logits_of(400, 20000, BF)
    few, many = score(z[:4], None, 50), score(z, None, 50)
    assert torch.equal(few["top_ids"], many["top_ids"][:4])
    for x in ("lse", "entropy", "top_logp"):
        assert ((few[x] - many[x][:4]).nan_to_num().abs() <= 3e-5 + 2.0 ** -22 * many[x][:4].abs().nan_to_num()).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [64, 1025, 4096])
def test_gains_that_start_anywhere(d, dtype):
    x, dy = matrix(6, d, dtype).contiguous(), matrix(6, d, dtype, seed=4).contiguous()
    gain, bias = matrix(1, d + 1, dtype, seed=1, mean=1.0)[0].contiguous(), matrix(1, d + 3, dtype, seed=2)[0].contiguous()
    y, mean, rstd = forward(x, gain[1:], bias[3:])
    want = torch.nn.functional.layer_norm(x.double(), (d,), gain[1:].double(), bias[3:].double(), EPS)
    assert ((y.double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + 2e-5 * (1 + want.abs())).all()
    other = gradients(x, dy, gain[1:].clone(), mean, rstd)
    for a, b in zip(gradients(x, dy, gain[1:], mean, rstd), other):
        assert ((a.double() - b.double()).abs() <= torch.finfo(dtype).eps * b.double().abs() + 2e-5 * b.double().abs().max()).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d", [(600, 127), (600, 129), (4, 255), (4, 257), (600, 511), (600, 513), (593, 1023), (592, 1537), (591, 1537), (600, 8191)])
def test_norms_of_rows_that_start_anywhere(n, d, dtype):
    """where a thread has another number of columns, and a warp its first or last"""
    norms.test_forward(n, d, 0, 0, 0.5, dtype)
    norms.test_backward(n, d, 3, 1, True, dtype)


def test_one_workspace_for_calls_in_turn():
    """a call leaves nothing in it that the next minds, whatever it held"""
    n, V, d = 500, 900, 40
    ids = torch.randint(V, (n,), device="cuda")
    dy = matrix(n, d, BF)
    need = max(B.embedding_backward_workspace_bytes(n, V, d), B.layernorm_workspace_bytes(n, d), 4096)
    ws = torch.randint(256, (need,), dtype=torch.uint8, device="cuda")
    first = torch.empty(V, d, device="cuda")
    B.embedding_backward(dy, ids, first, ws)
    x = matrix(n, d, BF)
    _, mean, rstd = forward(x, None, None)
    B.layernorm_backward(dy, x, None, mean, rstd, d_gain=torch.empty(d, device="cuda"), workspace=ws)
    B.embedding_forward(dy, torch.full((3,), 10 ** 6, device="cuda"), torch.empty(3, d, device="cuda", dtype=BF), ws)
    assert B.last_device_status(ws) == B.E_BAD_LABEL
    again = torch.empty(V, d, device="cuda")
    B.embedding_backward(dy, ids, again, ws)
    assert torch.equal(first, again) and B.last_device_status(ws) == B.OK


@pytest.mark.parametrize("dtype", [F32, BF])
def test_vocabularies_beyond_a_clusters_shared_memory(dtype):
    z = logits_of(2, 1_000_003, dtype)
    for tail in (False, True):
        ids, values = teacher(z, 40, 1.0, tail)
        check_distill(z, ids, values, None, 1.0, tail)


def test_in_a_process_with_guards():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert not GUARDED
    sel = ["tests/test_gpu_layernorm.py::test_backward", "tests/test_gpu_embedding.py::test_gradient", "tests/test_gpu_embedding.py::test_gradient_of_crowds",
           "tests/test_gpu_model_ends.py", "tests/test_gpu_logprobs.py::test_rows", "tests/test_gpu_distill.py::test_rows"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"] + sel, cwd=root,
                       env=dict(os.environ, STREAMBP_WS_GUARD="1"), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,V,d", [(1, 70000, 260), (9, 5000, 4099), (3000, 20011, 1001), (70000, 60, 33), (66000, 300001, 60)])
def test_embedding_gradients_that_overwrite_large_tables(n, V, d, dtype):
    """rows without tokens are cleared by other blocks than those of small tables: the first and last rows, tokens of every row"""
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(V, (n,), generator=g, device="cuda")
    ids[-1] = V - 1
    dy = matrix(n, d, dtype)
    out = torch.full((V, d), float("nan"), device="cuda")
    ws = B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, d))
    B.embedding_backward(dy, ids, out, ws)
    want = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, dy.double())
    size = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, dy.double().abs())
    assert B.last_device_status(ws) == B.OK
    # a row's sum is a chunk's values one after another, then the chunks' sums: fewer than 400 roundings
    assert ((out.double() - want).abs() <= 400 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d", [(4096, 8), (4097, 256), (5000, 264), (4099, 512), (9000, 384), (4100, 768), (4096, 776), (7001, 16)])
def test_norms_of_many_narrow_rows(n, d, dtype):
    """a warp's rows and a block's, the sums of a block's warps"""
    norms.test_backward(n, d, 0, 0, False, dtype)
    norms.test_backward(n, d, 8, 0, True, dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (31, 5, 40), (32, 1000, 2056), (33, 7, 33), (64, 3, 4099), (128, 1, 512), (128, 200, 96), (129, 4, 64)])
def test_embedding_gradients_of_few_tokens(n, V, d, accumulate, dtype):
    """tokens of one id across all words of the search, padding and ids outside the table among them"""
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(V, (n,), generator=g, device="cuda")
    if n > 8:
        ids[3], ids[n // 2], ids[n - 1] = -1, V, -1
    dy = matrix(n, d, dtype, 8, 0)
    start = matrix(V, d, F32, seed=9).contiguous()
    out = start.clone() if accumulate else torch.full((V, d), float("nan"), device="cuda")
    ws = B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, d))
    B.embedding_backward(dy, ids, out, ws, scale=0.5, padding_id=-1, accumulate=accumulate)
    assert B.last_device_status(ws) == (B.E_BAD_LABEL if n > 8 else B.OK)
    part = (ids >= 0) & (ids < V)
    sums = lambda x: torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids[part], x.double()[part])
    want = 0.5 * sums(dy) + (start.double() if accumulate else 0.0)
    # at most 130 roundings of the sum, one of the result
    assert ((out.double() - want).abs() <= 130 * 2.0 ** -25 * sums(dy.abs()) + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,d", [(3, 12288), (600, 9001), (450, 8200), (2, 16384), (2, 16385), (5, 16392), (200, 20488), (2, 32768), (2, 32776)])
def test_norms_of_wide_rows(n, d, dtype):
    """the widest rows that a block or a cluster of two or four holds, and the next"""
    norms.test_backward(n, d, 0, 0, False, dtype)
    norms.test_backward(n, d, 8, 0, True, dtype)
    norms.test_forward(n, d, 0, 0, 0.5, dtype)
    norms.test_forward(n, d, 8, 0, 30.0, dtype)


@pytest.mark.parametrize("n,V,d", [(50, 900, 64), (3000, 500, 72), (3000, 20011, 1000), (70000, 2000, 16)])
def test_embedding_gradients_captured_and_two_at_once(n, V, d):
    """replays read what is there then, and write every row; two of them run at the same time with workspaces of their own"""
    streams, calls = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        ids, dy = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, d, device="cuda")
        out, ws = torch.empty(V, d, device="cuda"), B.alloc_workspace(B.embedding_backward_workspace_bytes(n, V, d))
        B.embedding_backward(dy, ids, out, ws)                     # (attributes of the kernels are set outside the capture)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.embedding_backward(dy, ids, out, ws)
        calls.append((ids, dy, out, ws, graph))
    for round_ in range(3):
        for i, (ids, dy, out, ws, graph) in enumerate(calls):
            g = torch.Generator(device="cuda").manual_seed(10 * round_ + i)
            ids.copy_(torch.randint(V, (n,), generator=g, device="cuda") // (1 + 2 * round_))
            dy.copy_(torch.randn(n, d, generator=g, device="cuda"))
            out.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, call in zip(streams, calls):
            with torch.cuda.stream(s):
                call[4].replay()
        torch.cuda.synchronize()
        for ids, dy, out, ws, graph in calls:
            want = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, dy.double())
            size = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids, dy.double().abs())
            assert B.last_device_status(ws) == B.OK
            # fewer than 400 roundings to a row's sum (a chunk's values, then the chunks)
            assert ((out.double() - want).abs() <= 400 * 2.0 ** -24 * size).all()


def test_norm_gradients_two_at_once():
    streams, calls = [torch.cuda.Stream() for _ in range(2)], []
    for i, (n, d) in enumerate(((5000, 768), (900, 1537))):
        x, dy = matrix(n, d, BF, seed=i), matrix(n, d, BF, seed=7 + i)
        _, mean, rstd = forward(x, None, None)
        calls.append((x, dy, None, mean, rstd, gradients(x, dy, None, mean, rstd)))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, (x, dy, gain, mean, rstd, _) in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(gradients(x, dy, gain, mean, rstd))
        torch.cuda.synchronize()
        for a, call in zip(got, calls):
            assert all(torch.equal(x, y) for x, y in zip(a, call[5]))
