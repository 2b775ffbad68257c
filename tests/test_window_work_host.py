"""The geometry of the windowed backward on the CPU: every key's gradients are written once, by its owner or by the kernel that
joins segments, every visible pair is taken once, and no slot lies behind the workspace (window_work_check.cpp, compiled here
against the header that the kernels and the workspace query use)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("window") / "window_work_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2506_03077_b200", "csrc"),
                    os.path.join(ROOT, "tests", "window_work_check.cpp"), "-o", exe], check=True)
    return lambda *a: subprocess.run([exe, *map(str, a)], capture_output=True, text=True, timeout=600)


# n, q0, query heads, key heads, head_dim, window, sinks: the sink tiles are all the key tiles, the last of them a short one
@pytest.mark.parametrize("shape", [(20, 0, 16, 1, 64, 8, 1), (49, 50, 16, 1, 64, 8, 4), (71, 50, 16, 1, 128, 8, 100),
                                   (151, 50, 32, 8, 128, 64, 200), (100, 0, 28, 4, 128, 30, 1)])
def test_keys_behind_the_sink_tiles(check, shape):
    r = check("shape", *shape)
    assert r.returncode == 0, r.stdout


def test_sweep_of_shapes(check):
    r = check("sweep")
    assert r.returncode == 0, r.stdout[:2000]
