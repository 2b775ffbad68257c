"""Host-side refusals of the optimizer entry points (no GPU: arguments are checked before any CUDA call)."""
import ctypes as C

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from paper_2506_03077_b200 import build as build_mod

P = 0x10000     # an aligned address that is never read: every call here is refused on the host


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.lib()


def adamw(lib, tensor=None, n=1, grad_scale=None, device_step=None, **cfg):
    c = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, param_dtype=B.STREAMBP_BF16, state_dtype=B.STATE_F32, step=1)
    c.update(cfg)
    t = dict(param=P, master=None, grad=P, m=P, v=P, m_scale=None, v_scale=None, count=64, weight_decay=0.0)
    t.update(tensor or {})
    cc, tt = B.AdamWCfgC(**c), B.AdamWTensorC(**t)
    return lib.streambp_adamw_step(C.byref(cc), C.byref(tt), n, grad_scale, device_step, None)


@pytest.mark.parametrize("kw,status", [
    (dict(param_dtype=7), B.E_DTYPE), (dict(state_dtype=2), B.E_DTYPE), (dict(lr=-1.0), B.E_SHAPE),
    (dict(lr=float("nan")), B.E_SHAPE), (dict(lr=float("inf")), B.E_SHAPE), (dict(beta1=1.0), B.E_SHAPE),
    (dict(beta2=-0.1), B.E_SHAPE), (dict(beta2=float("nan")), B.E_SHAPE), (dict(eps=-1e-8), B.E_SHAPE),
    (dict(step=0), B.E_SHAPE), (dict(n=-1), B.E_SHAPE), (dict(grad_scale=P + 2), B.E_ALIGN),
    (dict(step=0, grad_scale=P + 1), B.E_SHAPE), (dict(step=0, device_step=P + 4), B.E_ALIGN),
    (dict(tensor=dict(param=None)), B.E_NULL), (dict(tensor=dict(grad=None)), B.E_NULL), (dict(tensor=dict(m=None)), B.E_NULL),
    (dict(tensor=dict(v=None)), B.E_NULL), (dict(tensor=dict(param=P + 8)), B.E_ALIGN), (dict(tensor=dict(grad=P + 4)), B.E_ALIGN),
    (dict(tensor=dict(m=P + 4)), B.E_ALIGN), (dict(tensor=dict(v=P + 4)), B.E_ALIGN), (dict(tensor=dict(master=P + 4)), B.E_ALIGN),
    (dict(tensor=dict(count=-1)), B.E_SHAPE), (dict(tensor=dict(weight_decay=-0.1)), B.E_SHAPE),
    (dict(tensor=dict(weight_decay=float("nan"))), B.E_SHAPE),
    (dict(param_dtype=B.STREAMBP_F32, tensor=dict(master=P)), B.E_DTYPE),
    (dict(state_dtype=B.STATE_MX8), B.E_NULL), (dict(state_dtype=B.STATE_MX8, tensor=dict(m_scale=P)), B.E_NULL),
])
def test_adamw_refusals(lib, kw, status):
    assert adamw(lib, **kw) == status


def test_adamw_of_nothing(lib):
    assert adamw(lib, n=0) == B.OK
    assert adamw(lib, tensor=dict(count=0, param=None, grad=None, m=None, v=None)) == B.OK
    assert lib.streambp_adamw_step(None, None, 0, None, None, None) == B.E_NULL


def test_grad_norm_refusals(lib):
    need = lib.streambp_grad_norm_workspace_bytes()
    def call(grad=P, count=8, n=1, most=1.0, norm=P, scale=P, ws=P, size=need):
        return lib.streambp_grad_norm((C.c_void_p * 1)(grad), (C.c_int64 * 1)(count), n, most, norm, scale, ws, size, None)
    assert call(norm=None) == B.E_NULL and call(ws=None) == B.E_NULL and call(grad=None) == B.E_NULL
    assert call(n=-1) == B.E_SHAPE and call(count=-1) == B.E_SHAPE
    assert call(most=0.0) == B.E_SHAPE and call(most=-1.0) == B.E_SHAPE and call(most=float("nan")) == B.E_SHAPE
    assert call(ws=P + 128) == B.E_ALIGN and call(norm=P + 2) == B.E_ALIGN and call(scale=P + 1) == B.E_ALIGN
    assert call(grad=P + 4) == B.E_ALIGN and call(size=need - 1) == B.E_WORKSPACE


def test_mx8_refusals(lib):
    assert lib.streambp_mx8_encode(P, -1, 0, P, P, None) == B.E_SHAPE and lib.streambp_mx8_decode(P, P, -1, P, 0, None) == B.E_SHAPE
    assert lib.streambp_mx8_encode(None, 8, 0, P, P, None) == B.E_NULL and lib.streambp_mx8_encode(P, 8, 0, P, None, None) == B.E_NULL
    assert lib.streambp_mx8_encode(P + 4, 8, 0, P, P, None) == B.E_ALIGN and lib.streambp_mx8_encode(P, 8, 0, P + 4, P, None) == B.E_ALIGN
    assert lib.streambp_mx8_decode(P, P, 8, None, 0, None) == B.E_NULL and lib.streambp_mx8_decode(P, P, 8, P, 5, None) == B.E_DTYPE
    assert lib.streambp_mx8_decode(P, P, 8, P + 2, 1, None) == B.E_ALIGN and lib.streambp_mx8_decode(P + 1, P, 8, P, 1, None) == B.E_ALIGN
    assert lib.streambp_mx8_encode(None, 0, 0, None, None, None) == B.OK and lib.streambp_mx8_decode(None, None, 0, None, 0, None) == B.OK


def test_plan_refuses_host_tensors():
    t = {k: torch.zeros(8) for k in ("param", "grad", "m", "v")}
    with pytest.raises(ValueError):
        B.AdamWPlan([t])
    with pytest.raises(ValueError):
        B.AdamWPlan([])


def epilogue(lib, **kw):
    a = dict(A=P, lda=64, W=P, ldw=64, M=16, N=32, K=64, bias=P, act=3, residual=P + 0x1000, ldr=32, C=P, ldc=32, pre=P + 0x2000,
             ldp=32, dtype=B.STREAMBP_BF16)
    a.update(kw)
    return lib.streambp_gemm_epilogue(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(A=None), B.E_NULL), (dict(W=None), B.E_NULL), (dict(C=None), B.E_NULL), (dict(dtype=2), B.E_DTYPE),
    (dict(M=0), B.E_SHAPE), (dict(N=0), B.E_SHAPE), (dict(K=0), B.E_SHAPE), (dict(M=1 << 31), B.E_SHAPE),
    (dict(act=-1), B.E_SHAPE), (dict(act=5), B.E_SHAPE), (dict(lda=63), B.E_SHAPE), (dict(ldw=1), B.E_SHAPE),
    (dict(ldc=31), B.E_SHAPE), (dict(ldr=31), B.E_SHAPE), (dict(ldp=31), B.E_SHAPE), (dict(A=P + 1), B.E_ALIGN),
    (dict(C=P + 1), B.E_ALIGN), (dict(bias=P + 1), B.E_ALIGN), (dict(residual=P + 1), B.E_ALIGN), (dict(pre=P + 3), B.E_ALIGN),
    (dict(dtype=B.STREAMBP_F32, W=P + 2), B.E_ALIGN), (dict(residual=P, ldr=40), B.E_SHAPE), (dict(pre=P), B.E_SHAPE),
    (dict(pre=P + 0x1000), B.E_SHAPE),
])
def test_gemm_epilogue_refusals(lib, kw, status):
    assert epilogue(lib, **kw) == status


def test_gemm_epilogue_backward_refusals(lib):
    need = lib.streambp_gemm_epilogue_workspace_bytes(16, 32)
    assert need > 0 and lib.streambp_gemm_epilogue_workspace_bytes(0, 32) == 0 and lib.streambp_gemm_epilogue_workspace_bytes(16, -1) == 0
    def call(dC=P, ldd=32, pre=P + 0x1000, ldp=32, act=4, M=16, N=32, dZ=P + 0x2000, ldz=32, dbias=P, acc=0, dtype=1, ws=P, size=need):
        return lib.streambp_gemm_epilogue_backward(dC, ldd, pre, ldp, act, M, N, dZ, ldz, dbias, acc, dtype, ws, size, None)
    assert call(dC=None) == B.E_NULL and call(pre=None) == B.E_NULL and call(dZ=None, dbias=None) == B.E_NULL and call(ws=None) == B.E_NULL
    assert call(dtype=3) == B.E_DTYPE and call(act=9) == B.E_SHAPE and call(M=0) == B.E_SHAPE and call(N=0) == B.E_SHAPE
    assert call(ldd=31) == B.E_SHAPE and call(ldp=31) == B.E_SHAPE and call(ldz=31) == B.E_SHAPE
    assert call(dC=P + 1) == B.E_ALIGN and call(dZ=P + 1) == B.E_ALIGN and call(dbias=P + 2) == B.E_ALIGN and call(ws=P + 64) == B.E_ALIGN
    assert call(size=need - 1) == B.E_WORKSPACE and call(dZ=P, ldz=40) == B.E_SHAPE and call(dZ=P + 0x1000, ldz=40) == B.E_SHAPE


def window_fwd(lib, **kw):
    a = dict(q=P, k=P, v=P, n=16, q0=8, Hq=4, Hkv=2, dh=64, dtype=B.STREAMBP_BF16, window=4, sinks=1, o=P, lse=P, engine=0)
    a.update(kw)
    return lib.streambp_attention_window_forward(*a.values(), None)


SIZES = [
    (dict(n=0), B.E_SHAPE), (dict(n=-1), B.E_SHAPE), (dict(q0=-1), B.E_SHAPE), (dict(n=1 << 31), B.E_SHAPE),
    (dict(q0=1 << 30), B.E_SHAPE), (dict(Hq=0), B.E_SHAPE), (dict(Hkv=3), B.E_SHAPE), (dict(Hkv=0), B.E_SHAPE), (dict(dh=96), B.E_SHAPE),
    (dict(window=0), B.E_SHAPE), (dict(window=-5), B.E_SHAPE), (dict(sinks=-1), B.E_SHAPE), (dict(dtype=2), B.E_DTYPE),
    (dict(Hq=1 << 17, Hkv=1 << 17), B.E_SHAPE),
]


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(q=None), B.E_NULL), (dict(k=None), B.E_NULL), (dict(v=None), B.E_NULL), (dict(o=None), B.E_NULL), (dict(lse=None), B.E_NULL),
    (dict(q=P + 8), B.E_ALIGN), (dict(k=P + 2), B.E_ALIGN), (dict(o=P + 4), B.E_ALIGN), (dict(lse=P + 2), B.E_ALIGN),
    (dict(engine=3), B.E_SHAPE), (dict(engine=-1), B.E_SHAPE), (dict(dtype=B.STREAMBP_F32, engine=2), B.E_DTYPE)])
def test_window_forward_refusals(lib, kw, status):
    assert window_fwd(lib, **kw) == status


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(d_o=None), B.E_NULL), (dict(dq=None), B.E_NULL), (dict(ws=None), B.E_NULL), (dict(dk=P + 8), B.E_ALIGN),
    (dict(ws=P + 16), B.E_ALIGN), (dict(size=100), B.E_WORKSPACE), (dict(grad=2), B.E_DTYPE), (dict(grad=1, acc=1), B.E_DTYPE),
    (dict(dtype=0, grad=1), B.E_DTYPE), (dict(engine=3), B.E_SHAPE), (dict(dtype=0, engine=2), B.E_DTYPE)])
def test_window_backward_refusals(lib, kw, status):
    a = dict(q=P, k=P, v=P, o=P, d_o=P, lse=P, n=16, q0=8, Hq=4, Hkv=2, dh=64, dtype=B.STREAMBP_BF16, window=4, sinks=1, grad=0, acc=0,
             dq=P, dk=P, dv=P, ws=P, size=1 << 20, engine=0)
    a.update(kw)
    assert lib.streambp_attention_window_backward(*a.values(), None) == status


def test_window_workspace(lib):
    size = lib.streambp_attention_window_workspace_bytes
    assert size(16, 8, 4, 2, 64, 4, 1) > 0 and size(16, 8, 4, 2, 96, 4, 1) == 0 and size(16, 8, 4, 3, 64, 4, 1) == 0
    assert size(0, 8, 4, 2, 64, 4, 1) == 0 and size(16, 8, 4, 2, 64, 0, 1) == 0
    # what the sinks' segments take is bounded, however many sinks there are
    assert all(size(32768, 0, 32, 8, 128, 128, s) < (200 << 20) for s in (0, 1, 4, 128, 1000, 16000, 32767, 1 << 20))


def _key_work(n, q0, Hkv, window, sinks, TK, TQ, wsegs):
    """The key tiles' work as window.cuh lays it out, restated: (key tile, query tiles, segment) of every item."""
    kv, qt = q0 + n, -(-n // TQ)
    lo = max(0, q0 - window + 1) // TK
    st = min(-(-sinks // TK), -(-kv // TK))
    length = (window + TK + 2 * TQ - 2) // TQ
    walk = min(length, qt)
    wlen = -(-walk // wsegs) if wsegs > 1 else length
    length = wlen if wsegs > 1 else max(8, length)
    segs = -(-qt // length) if st else 1
    most = 592 // min(592, st * Hkv) if st else 1
    if segs > most:
        length = -(-qt // most)
        segs = -(-qt // length)
    first = lambda kt: (kt * TK - q0) // TQ if kt * TK > q0 else 0
    items = []
    for kt in list(range(st)) + list(range(max(st, lo), -(-kv // TK))):
        last = kt * TK + TK - 1 + window - 1 - q0
        n_seg, step = (segs, length) if kt < st else (wsegs, wlen)
        end = qt if kt < st else (min(qt, last // TQ + 1) if last >= 0 else 0)
        for s in range(n_seg):
            b = first(kt) + s * step
            items.append((kt, range(b, end if n_seg == 1 else min(end, b + step)), s if n_seg > 1 else -1))
    return items


def test_key_work_covers_every_visible_pair_once():
    """Every visible (query, key) pair lies in exactly one item; where windows are not cut, only sinks are seen behind the
    first segment of a sink tile."""
    import random
    rng = random.Random(0)
    for _ in range(700):
        TK, TQ = rng.choice(((4, 4), (8, 8), (8, 4), (16, 4), (16, 3), (8, 1)))
        n, q0 = rng.randrange(1, 120), rng.choice((0, rng.randrange(0, 80)))
        window, sinks = rng.randrange(1, 60), rng.choice((0, 1, 3, 5, 17, 40))
        kv = q0 + n
        window = min(window, kv)
        sinks = min(sinks, kv)
        if sinks == kv or window == kv:
            window, sinks = kv, 0
        walk = min((window + TK + 2 * TQ - 2) // TQ, -(-n // TQ))
        wsegs = rng.choice([s for s in (1, 1, 2, 4, 8) if s <= walk])
        seen = {}
        for kt, tiles, seg in _key_work(n, q0, rng.choice((1, 8, 200)), window, sinks, TK, TQ, wsegs):
            for qt in tiles:
                assert 0 <= qt < -(-n // TQ)
                for t in range(q0 + qt * TQ, min(q0 + n, q0 + qt * TQ + TQ)):
                    for j in range(kt * TK, min(kv, kt * TK + TK)):
                        if j <= t and (t - j < window or j < sinks):
                            seen[(t, j)] = seen.get((t, j), 0) + 1
                            assert seg <= 0 or wsegs > 1 or j < sinks
        want = {(t, j) for t in range(q0, kv) for j in range(t + 1) if t - j < window or j < sinks}
        assert set(seen) == want and set(seen.values()) <= {1}
