"""The product with bias, activation and residual in its epilogue, and the gradient of that epilogue, against numpy in
64 bits.

Bounds: the operands are multiplied exactly and summed in fp32, K terms: at most K 2^-24 of the sum of the terms'
magnitudes (tensor cores add in fewer, wider steps; the bound holds for any order).  An activation with slope at most
1.13 passes that on and adds its own error of at most 2^-19 of max(1, |z|) (ex2.approx and rcp.approx: 2^-21 in total,
tanh through the sigmoid of 2a with |2a| <= 2^7 before it saturates); bf16 results are rounded once, 2^-8."""
import math

import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
E32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
FENCE = 7.0


def act64(z, act):
    if act == "relu":
        return np.maximum(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + np.vectorize(math.erf, otypes=[float])(z / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).astype(float)
    if act == "gelu":
        return 0.5 * (1 + np.vectorize(math.erf, otypes=[float])(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = np.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def rand(seed, *shape, std=1.0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def padded(x, extra):
    """`x` as a view of rows `extra` elements apart, with a fence behind every row and behind the matrix."""
    buf = torch.full((x.shape[0] + 1, x.shape[1] + extra), FENCE, dtype=x.dtype, device="cuda")
    view = buf[:-1, :x.shape[1]]
    view.copy_(x)
    return view, buf


def fence_ok(buf, cols):
    return bool((buf[:-1, cols:] == FENCE).all()) and bool((buf[-1] == FENCE).all())


def f64(t):
    return t.double().cpu().numpy()


def check_forward(M, N, K, act, dtype, bias=True, residual=True, pre=True, extra=8, seed=0):
    A, W = rand(seed, M, K, dtype=dtype), rand(seed + 1, N, K, std=K ** -0.5, dtype=dtype)
    b = rand(seed + 2, N, dtype=dtype) if bias else None
    R, rbuf = padded(rand(seed + 3, M, N, dtype=dtype), extra) if residual else (None, None)
    Z, zbuf = padded(torch.zeros(M, N, dtype=dtype, device="cuda"), 2 * extra) if pre else (None, None)
    Y, ybuf = padded(torch.zeros(M, N, dtype=dtype, device="cuda"), extra)
    B.gemm_epilogue(A, W, Y, bias=b, activation=act, residual=R, pre=Z)
    assert B.last_launch_count() == 1
    a64, w64 = f64(A), f64(W)
    z = a64 @ w64.T + (f64(b) if bias else 0)
    ez = (K + 1) * E32 * (np.abs(a64) @ np.abs(w64).T + (np.abs(f64(b)) if bias else 0))
    y = act64(z, act) + (f64(R) if residual else 0)
    ey = 1.13 * ez + (2.0 ** -19 * np.maximum(1, np.abs(z)) if act not in ("none", "relu") else 0) + 2 * E32 * np.abs(y)
    h = HALF[dtype]
    assert (np.abs(f64(Y) - y) <= ey + h * (np.abs(y) + ey)).all()
    assert fence_ok(ybuf, N)
    if pre:
        assert (np.abs(f64(Z) - z) <= ez + h * (np.abs(z) + ez)).all()
        assert fence_ok(zbuf, N)
    if residual:
        assert fence_ok(rbuf, N)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forward_every_activation(act, dtype):
    check_forward(200, 328, 136, act, dtype)


@pytest.mark.parametrize("M,N,K", [(1, 1, 8), (1, 256, 64), (3, 40, 8), (128, 256, 64), (129, 257, 72), (255, 31, 200),
                                   (257, 520, 1000), (300, 1027, 64), (64, 2000, 24)])
@pytest.mark.parametrize("bias,residual,pre", [(True, True, True), (False, False, False), (True, False, True)])
def test_forward_sizes(M, N, K, bias, residual, pre):
    check_forward(M, N, K, "gelu_tanh", torch.bfloat16, bias, residual, pre)


@pytest.mark.parametrize("extra", [0, 1, 4, 16])
def test_forward_leading_dimensions(extra):
    check_forward(130, 300, 64, "silu", torch.bfloat16, extra=extra)
    check_forward(66, 70, 33, "silu", torch.float32, extra=extra)


@pytest.mark.parametrize("K", [1, 7, 33, 100])
def test_forward_operands_outside_the_tensor_core_rules(K):
    """K is the dense leading dimension of A and W: not a multiple of 8 runs on CUDA cores."""
    check_forward(70, 90, K, "gelu", torch.bfloat16)


def test_forward_operands_with_padding_and_unaligned_start():
    A = rand(0, 50, 72, dtype=torch.bfloat16)[:, :64]
    W = rand(1, 60, 80, dtype=torch.bfloat16)[:, 3:67]          # starts on a 6-byte boundary: CUDA cores
    W2 = rand(1, 60, 80, dtype=torch.bfloat16)[:, 8:72]
    for w in (W, W2):
        Y = torch.zeros(50, 60, dtype=torch.bfloat16, device="cuda")
        B.gemm_epilogue(A, w, Y)
        y = f64(A) @ f64(w).T
        e = 64 * E32 * (np.abs(f64(A)) @ np.abs(f64(w)).T)
        assert (np.abs(f64(Y) - y) <= e + 2.0 ** -8 * (np.abs(y) + e)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_residual_may_be_the_output(dtype):
    A, W, b = rand(0, 150, 64, dtype=dtype), rand(1, 200, 64, dtype=dtype), rand(2, 200, dtype=dtype)
    R = rand(3, 150, 200, dtype=dtype)
    Y, Z = torch.zeros_like(R), R.clone()
    B.gemm_epilogue(A, W, Y, bias=b, activation="gelu", residual=R)
    B.gemm_epilogue(A, W, Z, bias=b, activation="gelu", residual=Z)
    assert torch.equal(Y, Z)


def test_activations_at_the_ends_of_the_range():
    """z from -3e4 to 3e4 through an identity product: no infinity or NaN, and the limits 0 and z."""
    z = torch.tensor([-3e4, -1e3, -100.0, -20.0, -8.0, 0.0, 8.0, 20.0, 100.0, 1e3, 3e4], device="cuda").to(torch.bfloat16)
    n = z.numel()
    eye = torch.eye(n, 16, device="cuda", dtype=torch.bfloat16)
    W = torch.zeros(n, 16, device="cuda", dtype=torch.bfloat16)
    W[:, 0] = z
    A = torch.zeros(1, 16, device="cuda", dtype=torch.bfloat16)
    A[0, 0] = 1
    del eye
    for act in ACTS:
        for dt in (torch.bfloat16, torch.float32):
            Y = torch.zeros(1, n, device="cuda", dtype=dt)
            B.gemm_epilogue(A.to(dt), W.to(dt), Y, activation=act)
            ref = act64(f64(z)[None], act)
            assert np.isfinite(f64(Y)).all()
            assert (np.abs(f64(Y) - ref) <= 2.0 ** -19 * np.maximum(1, np.abs(f64(z))) + HALF[dt] * np.abs(ref)).all()
            dz = torch.zeros_like(Y)
            B.gemm_epilogue_backward(torch.ones_like(Y), z[None].to(dt).contiguous(), act, dz)
            ref = slope64(f64(z)[None], act)
            assert (np.abs(f64(dz) - ref) <= 2.0 ** -18 + HALF[dt] * np.abs(ref)).all()


def test_large_offsets():
    """Rows whose element offsets pass 2^31: the last rows of a matrix with a large leading dimension."""
    M, ld = 300, 8_000_000
    buf = torch.zeros(M * ld, dtype=torch.bfloat16, device="cuda").view(M, ld)
    Y = buf[:, :64]
    A, W = rand(0, M, 64, dtype=torch.bfloat16), rand(1, 64, 64, dtype=torch.bfloat16)
    want = torch.zeros(M, 64, dtype=torch.bfloat16, device="cuda")
    B.gemm_epilogue(A, W, want, activation="relu")
    B.gemm_epilogue(A, W, Y, activation="relu")
    assert torch.equal(Y, want)
    dz = torch.zeros_like(want)
    B.gemm_epilogue_backward(Y, Y, "relu", dz)
    assert torch.equal(dz, torch.where(want > 0, want, torch.zeros_like(want)))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,extra", [(1, 1, 0), (1, 300, 0), (33, 8, 8), (200, 67, 3), (1000, 520, 8), (70, 2731, 0), (2100, 64, 0)])
def test_backward(act, dtype, M, N, extra):
    D, dbuf = padded(rand(0, M, N, dtype=dtype), extra)
    Z, _ = padded(rand(1, M, N, dtype=dtype) * 2, 2 * extra)
    G, gbuf = padded(torch.zeros(M, N, dtype=dtype, device="cuda"), extra)
    db = torch.full((N + 16,), FENCE, device="cuda")
    need = B.gemm_epilogue_workspace_bytes(M, N)
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    B.gemm_epilogue_backward(D, Z, act, G, db[:N], ws[:need])
    d64, s64 = f64(D), slope64(f64(Z), act)
    ref = d64 * s64
    es = 0 if act in ("none", "relu") else 2.0 ** -18
    e = es * np.abs(d64) + 2 * E32 * np.abs(ref)
    assert (np.abs(f64(G) - ref) <= e + HALF[dtype] * (np.abs(ref) + e)).all()
    # column sums of the unrounded values in fp32: any order of M additions
    eb = e.sum(0) + M * E32 * np.abs(ref).sum(0)
    assert (np.abs(f64(db[:N]) - ref.sum(0)) <= eb).all()
    assert fence_ok(gbuf, N) and fence_ok(dbuf, N) and bool((db[N:] == FENCE).all()) and bool((ws[need:] == 7).all())
    first = db.clone()
    B.gemm_epilogue_backward(D, Z, act, None, db[:N], ws[:need], accumulate=True)      # sums only, added
    assert torch.equal(db[:N], first[:N] + first[:N])
    B.gemm_epilogue_backward(D, None if act == "none" else Z, act, D)                   # dZ over dC, no sums
    assert torch.equal(D, G)


@pytest.mark.parametrize("M,N,ld,shift", [(2100, 63, 63, 0), (2100, 64, 65, 0), (2100, 64, 64, 1), (2100, 128, 129, 1), (2101, 191, 191, 1),
                                         (2049, 1001, 1001, 0), (2049, 1002, 1002, 0), (2049, 1002, 1003, 1), (300, 15001, 15001, 0), (2100, 1, 1, 1),
                                         (5000, 2, 3, 0)])
def test_backward_of_rows_that_start_anywhere(M, N, ld, shift):
    """bf16 rows of odd length or pitch, from an odd element on: the first and the last columns, and what lies around them."""
    def place(x):
        buf = torch.full((M * ld + shift + 64,), FENCE, dtype=torch.bfloat16, device="cuda")
        view = buf[shift:shift + M * ld].as_strided((M, N), (ld, 1))
        view.copy_(x)
        return view, buf
    D, _ = place(rand(0, M, N, dtype=torch.bfloat16))
    Z, _ = place(rand(1, M, N, dtype=torch.bfloat16) * 2)
    G, gbuf = place(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"))
    db = torch.full((N + 16,), FENCE, device="cuda")
    need = B.gemm_epilogue_workspace_bytes(M, N)
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    B.gemm_epilogue_backward(D, Z, "silu", G, db[:N], ws[:need])
    d64, s64 = f64(D), slope64(f64(Z), "silu")
    ref = d64 * s64
    e = 2.0 ** -18 * np.abs(d64) + 2 * E32 * np.abs(ref)
    assert (np.abs(f64(G) - ref) <= e + HALF[torch.bfloat16] * (np.abs(ref) + e)).all()
    assert (np.abs(f64(db[:N]) - ref.sum(0)) <= e.sum(0) + M * E32 * np.abs(ref).sum(0)).all()
    outside = torch.ones_like(gbuf, dtype=torch.bool)
    outside[shift:shift + M * ld].as_strided((M, N), (ld, 1)).fill_(False)
    assert bool((gbuf[outside] == FENCE).all()) and bool((db[N:] == FENCE).all()) and bool((ws[need:] == 7).all())
    first = db.clone()
    B.gemm_epilogue_backward(D, Z, "silu", None, db[:N], ws[:need])
    assert torch.equal(db, first)
    B.gemm_epilogue_backward(D, Z, "silu", D)
    assert torch.equal(D, G)


def test_gradient_against_differences():
    """sum(C * D) as a function of z: the backward's dZ against central differences of the forward in fp32."""
    M, N, h = 5, 40, 2.0 ** -6
    D, Z = rand(0, M, N), rand(1, M, N) * 2
    eye = torch.eye(N, device="cuda")
    for act in ACTS:
        ys = []
        for s in (+1, -1):
            Y = torch.zeros(M, N, device="cuda")
            B.gemm_epilogue(Z + s * h, eye, Y, activation=act)
            ys.append(Y.double())
        dz = torch.zeros(M, N, device="cuda")
        B.gemm_epilogue_backward(D, Z, act, dz)
        diff = (ys[0] - ys[1]) / (2 * h) * D.double()
        # third derivatives of these activations are below 2 where they are smooth; relu's kink is left out
        smooth = (Z.abs() > 2 * h) if act == "relu" else torch.ones_like(Z, dtype=torch.bool)
        bound = D.double().abs() * (2 * h * h / 6 + 2.0 ** -18 / h)
        assert bool(((dz.double() - diff).abs() <= bound)[smooth].all())


def test_capture_and_other_stream():
    A, W = rand(0, 300, 512, dtype=torch.bfloat16), rand(1, 700, 512, dtype=torch.bfloat16)
    Y, Z, want = (torch.zeros(300, 700, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    db = torch.zeros(700, device="cuda")
    ws = B.alloc_workspace(B.gemm_epilogue_workspace_bytes(300, 700))
    B.gemm_epilogue(A, W, want, activation="silu")
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        B.gemm_epilogue(A, W, Y, activation="silu", pre=Z)
        B.gemm_epilogue_backward(Y, Z, "silu", Z, db, ws)
    Y.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, want)
    Y.zero_()
    torch.cuda.synchronize()
    B.gemm_epilogue(A, W, Y, activation="silu", stream=s)
    s.synchronize()
    assert torch.equal(Y, want)


def test_refusals_of_shapes():
    A, W, Y = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((8, 16), (24, 16), (8, 24)))
    for bad in (dict(C_out=Y[:, :23]), dict(C_out=Y.float()), dict(C_out=Y.t()), dict(bias=Y[0, :23]), dict(residual=Y[:7]),
                dict(pre=Y.float()), dict(W=W[:, :8]), dict(C_out=Y.cpu())):
        kw = dict(A=A, W=W, C_out=Y)
        kw.update(bad)
        with pytest.raises(ValueError):
            B.gemm_epilogue(**kw)
    with pytest.raises(KeyError):
        B.gemm_epilogue(A, W, Y, activation="swish")
    with pytest.raises(B.StreamBPError):
        B.gemm_epilogue(A, W, Y, pre=Y)
    with pytest.raises(B.StreamBPError):
        B.gemm_epilogue_backward(Y, Y, "silu", Y, torch.zeros(24, device="cuda"))       # no workspace
