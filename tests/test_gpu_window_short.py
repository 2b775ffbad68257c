"""Windowed backward of short sequences whose sink tiles are all of their key tiles, the last a short one, with the work of
those tiles cut into segments: all rows of dk and dv in every gradient mode, against numpy in 64 bits (bounds as in
test_gpu_window.py)."""
import pytest
import torch

from test_gpu_window import BF, Case, F32, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n,q0,window,sinks", [
    (16, 1, 20, 0, 8, 1), (16, 1, 17, 0, 8, 1), (16, 1, 49, 50, 8, 4), (16, 1, 71, 50, 8, 100), (16, 1, 100, 0, 100, 99),
    (32, 8, 151, 50, 64, 200), (28, 4, 100, 0, 30, 1), (12, 4, 127, 0, 1, 3), (4, 2, 333, 0, 40, 300), (47, 1, 60, 199, 33, 257)])
def test_sink_tiles_are_all_the_tiles(Hq, Hkv, n, q0, window, sinks, dh):
    run(Case(n, q0, Hq, Hkv, dh, window, sinks), grads=(F32, BF))       # overwriting a prefill of NaN, and adding to fp32
