"""The workspace guards of the debug mode around the windowed backward and the epilogue's gradient."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_epilogue import FENCE, padded, rand
from test_gpu_window import BF, Case, F32

pytestmark = pytest.mark.gpu

GUARDED = "STREAMBP_WS_GUARD" in os.environ       # read by the library once per process: below, in one of its own


def armed(ws, fill):
    """Whether something wrote the last 256 bytes of a workspace, which hold the guard behind its last buffer, if there are guards."""
    return not GUARDED or bool((ws[-256:] != fill).any())


@pytest.mark.parametrize("dtype,engine", [(BF, 0), (BF, 1), (F32, 0)])
@pytest.mark.parametrize("n,q0,Hq,Hkv,dh,window,sinks", [
    (1500, 0, 2, 1, 64, 100, 3), (300, 200, 4, 2, 128, 64, 0), (49, 50, 16, 1, 64, 8, 4), (777, 100, 32, 32, 128, 90, 3)])
def test_windowed_backward(n, q0, Hq, Hkv, dh, window, sinks, dtype, engine):
    c = Case(n, q0, Hq, Hkv, dh, window, sinks, dtype)
    o, lse = c.forward(engine)
    need = B.attention_window_workspace_bytes(n, q0, Hq, Hkv, dh, window, sinks)
    for gd in (F32, BF) if dtype == BF else (F32,):
        ws = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
        out = [torch.empty_like(x, dtype=gd) for x in (c.q, c.k, c.v)]
        B.attention_window_backward(c.q, c.k, c.v, o, c.do, lse, q0, window, sinks, *out, ws, engine=engine)
        assert B.last_device_status(ws) == B.OK and armed(ws, 7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,extra", [(1, 1, 0), (333, 2731, 0), (2100, 64, 0), (2049, 1001, 0), (2048, 4096, 8), (5000, 2, 1)])
def test_epilogue_gradient(M, N, extra, dtype):
    D, _ = padded(rand(0, M, N, dtype=dtype), extra)
    Z, _ = padded(rand(1, M, N, dtype=dtype), extra)
    db = torch.full((N + 16,), FENCE, device="cuda")
    ws = torch.full((B.gemm_epilogue_workspace_bytes(M, N),), 7, dtype=torch.uint8, device="cuda")
    B.gemm_epilogue_backward(D, Z, "silu", torch.empty_like(D), db[:N], ws)
    assert B.last_device_status(ws) == B.OK and armed(ws, 7) and bool((db[N:] == FENCE).all())
    B.gemm_epilogue_backward(D, Z, "silu", torch.empty_like(D))              # no sums: no workspace


def test_in_a_process_with_guards():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, STREAMBP_WS_GUARD="1")
    assert not GUARDED
    sel = [f"tests/test_gpu_operator_guards.py::{t}" for t in ("test_windowed_backward", "test_epilogue_gradient")]
    sel += ["tests/test_gpu_window_short.py", "tests/test_gpu_window.py::test_sink_sums_joined_from_segments",
            "tests/test_gpu_window.py::test_head_layouts", "tests/test_gpu_epilogue.py::test_backward"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"] + sel, cwd=root, env=env,
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
