"""AdamW over many tensors, the norm of all gradients and the 8-bit form of the moments against numpy in 64 bits.

Bounds: a rounding to fp32 is off by at most 2^-24 of the value, to bf16 by 2^-8, to e4m3 by 2^-4 (below the smallest
normal code, 2^-6, by half of the smallest code, 2^-10)."""
import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu

H = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)
E32, FENCE = 2.0 ** -24, 77


def f32(x):
    return float(np.float32(x))


class Case:
    """Tensors of the given sizes inside larger buffers, with a fence of known values behind each."""

    def __init__(self, sizes, param=torch.bfloat16, mx8=False, master=False, seed=0, grad_std=1e-2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda n, std=1.0: torch.randn(n, generator=g, device="cuda") * std
        self.buffers, self.tensors, self.mx8 = [], [], mx8
        for i, n in enumerate(sizes):
            t = {"param": self.fenced(rand(n, 0.02).to(param)), "grad": self.fenced(rand(n, grad_std)),
                 "weight_decay": 0.1 * (i % 2)}
            if master:
                t["master"] = self.fenced(t["param"].float() * (1 + 1e-3))
            m, u = rand(n, 1e-3), rand(n, 1e-3).abs()
            if mx8:
                nb = (n + 31) // 32
                for k, x in (("m", m), ("v", u)):
                    t[k] = self.fenced(torch.zeros(n, dtype=torch.uint8, device="cuda"))
                    t[k + "_scale"] = self.fenced(torch.ones(nb, dtype=torch.uint8, device="cuda"))
                    B.mx8_encode(x, t[k], t[k + "_scale"], keep_nonzero=k == "v")
            else:
                t["m"], t["v"] = self.fenced(m), self.fenced(u * u)
            self.tensors.append(t)
        self.plan = B.AdamWPlan(self.tensors)

    def fenced(self, x):
        buf = torch.full((x.numel() + 64,), FENCE, dtype=x.dtype, device="cuda")
        view = buf[:x.numel()]
        view.copy_(x)
        self.buffers.append((buf, x.numel()))
        return view

    def check_fences(self):
        for buf, n in self.buffers:
            assert bool((buf[n:].float() == FENCE).all())

    def values(self, t, k):
        if not self.mx8:
            return t[k].double().cpu().numpy()
        out = torch.empty(t[k].numel(), device="cuda")
        B.mx8_decode(t[k], t[k + "_scale"], out)
        return out.double().cpu().numpy() ** (2 if k == "v" else 1)

    def state(self):
        return [{**{k: t[k].clone() for k in t if isinstance(t[k], torch.Tensor)}, "wd": t["weight_decay"],
                 "m64": self.values(t, "m"), "v64": self.values(t, "v")} for t in self.tensors]

    def bits(self):
        return [x.clone() for t in self.tensors for k, x in sorted(t.items()) if isinstance(x, torch.Tensor)]


def block_scale(x):
    """Upper bound of the power of two of each value's block of 32."""
    pad = np.zeros((len(x) + 31) // 32 * 32)
    pad[:len(x)] = np.abs(x)
    top = pad.reshape(-1, 32).max(1) * (1 + 1e-5)
    s = np.exp2(np.maximum(np.floor(np.log2(np.maximum(top, 1e-300))) - 7, -126))
    return np.repeat(s, 32)[:len(x)]


def check_step(case, before, step, gs=1.0, h=H):
    # taken in double by the call, which rounds each of beta, 1 - beta and the rates once: what a term's bound counts for its
    # constant.  (In 32 bits 1 - 0.95 would be 5e-7 off, relatively, before any of it.)
    lr, b1, b2, eps = (h[k] for k in ("lr", "beta1", "beta2", "eps"))
    for t, old in zip(case.tensors, before):
        g = old["grad"].double().cpu().numpy() * gs
        m = b1 * old["m64"] + (1 - b1) * g
        v = b2 * old["v64"] + (1 - b2) * g * g
        # three roundings of a term, one of the sum, one of the scaled gradient
        em = 5 * E32 * (np.abs(b1 * old["m64"]) + np.abs((1 - b1) * g))
        # the squared gradient: three roundings of its factor count twice, the product and the sum once
        ev = 8 * E32 * v
        p0 = old["master" if "master" in old else "param"].double().cpu().numpy()
        root = np.sqrt(v)
        den = root / np.sqrt(1 - b2 ** step) + eps
        rate = lr / (1 - b1 ** step)
        move = rate * m / den
        p = p0 * (1 - lr * f32(old["wd"])) - move
        # v and its root 7/2 + 2, the two constants 2, the sum 1, the quotient 4, the product 1, the moment em
        ep = 16 * E32 * np.abs(move) + rate / den * em + 4 * E32 * np.abs(p0) + E32 * np.abs(p)
        got = t["param"].double().cpu().numpy()
        if "master" in t:
            ma = t["master"].double().cpu().numpy()
            assert (np.abs(ma - p) <= ep).all()
            assert np.array_equal(got, t["master"].to(torch.bfloat16).double().cpu().numpy())
        else:
            assert (np.abs(got - p) <= ep + (2.0 ** -8 * (np.abs(p) + ep) if t["param"].dtype == torch.bfloat16 else 0)).all()
        gm, gv = case.values(t, "m"), case.values(t, "v")
        if not case.mx8:
            assert (np.abs(gm - m) <= em).all() and (np.abs(gv - v) <= ev).all()
        else:
            gu, eu = np.sqrt(gv), 6 * E32 * root
            assert (np.abs(gm - m) <= np.maximum(2.0 ** -4 * (np.abs(m) + em), 2.0 ** -10 * block_scale(m)) + em).all()
            # the root: rounded up to the smallest code where it would vanish
            su = block_scale(root)
            assert (np.abs(gu - root) <= np.maximum(2.0 ** -4 * (root + eu), 2.0 ** -9 * su) + eu).all()
            assert (gu[root > 0] > 0).all()
    case.check_fences()


SIZES = [1, 3, 31, 32, 33, 100, 4095, 4096, 4097, 100003]


@pytest.mark.parametrize("param,master", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("mx8", [False, True])
def test_step_matches_formula(param, master, mx8):
    c = Case(SIZES, param, mx8, master)
    gs = torch.tensor([0.37], device="cuda")
    for step in (1, 2, 9):
        before = c.state()
        B.adamw_step(c.plan, **H, step=step, grad_scale=gs)
        check_step(c, before, step, f32(0.37))


@pytest.mark.parametrize("n", [32, 33, 256, 257, 600])
def test_many_tensors(n):
    c = Case([(i * 37) % 211 + 1 for i in range(n)], torch.float32)
    before = c.state()
    B.adamw_step(c.plan, **H, step=3)
    assert B.last_launch_count() == (1 if n <= 256 else (n + 255) // 256)
    check_step(c, before, 3)


def test_empty_tensors_and_zero_state():
    c = Case([0, 5, 0, 64, 0], torch.bfloat16, mx8=True)
    for t in c.tensors:          # the documented start: zero codes, scale bytes of 1
        for k, v in (("m", 0), ("v", 0), ("m_scale", 1), ("v_scale", 1)):
            t[k].fill_(v)
    before = c.state()
    B.adamw_step(c.plan, **H, step=1)
    check_step(c, before, 1)
    only_empty = Case([0, 0], torch.float32)
    B.adamw_step(only_empty.plan, **H, step=1)


def test_gradients_of_very_different_sizes_in_a_block():
    """32 neighbours over 24 orders of magnitude: small roots stay above zero, so that the next step's quotient is
    bounded by the gradient's own size."""
    c = Case([64], torch.float32, mx8=True)
    t = c.tensors[0]
    for k, v in (("m", 0), ("v", 0), ("m_scale", 1), ("v_scale", 1)):
        t[k].fill_(v)
    t["grad"].copy_(torch.logspace(-20, 4, 64, device="cuda"))
    for step in (1, 2, 3):
        before = c.state()
        B.adamw_step(c.plan, **H, step=step)
        check_step(c, before, step)
    assert bool(torch.isfinite(t["param"]).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_step_is_left_out_when_the_scale_is_not_finite(bad):
    c = Case([100, 5000], torch.bfloat16, mx8=True)
    before = c.bits()
    B.adamw_step(c.plan, **H, step=1, grad_scale=torch.tensor([bad], device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(before, c.bits()))


def test_a_gradient_that_is_not_finite_marks_its_block_only():
    c = Case([96], torch.float32, mx8=True)
    t = c.tensors[0]
    t["grad"][40] = float("inf")
    B.adamw_step(c.plan, **H, step=1)
    m = torch.empty(96, device="cuda")
    B.mx8_decode(t["m"], t["m_scale"], m)
    assert bool(torch.isnan(m[32:64]).all()) and bool(torch.isfinite(m[:32]).all()) and bool(torch.isfinite(m[64:]).all())
    assert t["m_scale"].tolist()[1] == 255


def test_step_number_on_the_device_and_graph_replay():
    """A captured norm + step, replayed: the step number is read from the device at each replay."""
    a, b = Case(SIZES, torch.bfloat16, True), Case(SIZES, torch.bfloat16, True)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = [torch.zeros(1, device="cuda") for _ in range(4)]
    ws = [B.alloc_workspace(B.grad_norm_workspace_bytes()) for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        step.add_(1)
        B.grad_norm(a.plan, 0.5, out[0], out[1], ws[0])
        B.adamw_step(a.plan, **H, step=step, grad_scale=out[1])
    for k in range(1, 4):
        g.replay()
        B.grad_norm(b.plan, 0.5, out[2], out[3], ws[1])
        B.adamw_step(b.plan, **H, step=k, grad_scale=out[3])
        torch.cuda.synchronize()
        assert out[0].item() == out[2].item() and out[1].item() == out[3].item()
        for x, y in zip(a.state(), b.state()):
            assert np.allclose(x["m64"], y["m64"]) and np.allclose(x["v64"], y["v64"])
            # the constants are formed by the host's pow on one side, the device's on the other: 1 ulp of the move
            assert torch.allclose(x["param"].float(), y["param"].float(), rtol=2.0 ** -7, atol=1e-7)


def test_other_stream():
    c = Case([5000], torch.float32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    before = c.state()
    torch.cuda.synchronize()
    B.adamw_step(c.plan, **H, step=1, stream=s)
    s.synchronize()
    check_step(c, before, 1)


@pytest.mark.parametrize("sizes", [[1], [5, 0, 32769], [(i * 37) % 211 + 1 for i in range(1200)], [3_000_001, 17]])
def test_grad_norm(sizes):
    c = Case(sizes, torch.float32)
    ws = B.alloc_workspace(B.grad_norm_workspace_bytes() + 256)
    ws.fill_(FENCE)
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ref = np.sqrt(sum((t["grad"].double() ** 2).sum().item() for t in c.tensors))
    for most in (ref * 0.25, ref * 4):
        B.grad_norm(c.plan, most, norm, scale, ws[:-256])
        # eight squares and their sum in fp32: nine roundings of the sum, half of that for its root, one of the result
        assert abs(norm.item() - ref) <= 6 * E32 * ref
        want = min(1.0, f32(most) / (ref + 1e-6))
        assert abs(scale.item() - want) <= 8 * E32 * want
    first = norm.clone()
    B.grad_norm(c.plan, 1.0, norm, None, ws[:-256])
    assert torch.equal(first, norm) and bool((ws[-256:] == FENCE).all()) and B.last_device_status(ws) == B.OK


def test_grad_norm_of_huge_tiny_and_broken_gradients():
    c = Case([1000], torch.float32)
    ws = B.alloc_workspace(B.grad_norm_workspace_bytes())
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    g = c.tensors[0]["grad"]
    for size in (1e30, 1e-30, 1e-20, 1e-14):
        g.fill_(size)
        B.grad_norm(c.plan, 1.0, norm, scale, ws)
        ref = f32(size) * np.sqrt(1000.0)
        assert abs(norm.item() - ref) <= 6 * E32 * ref
    g[999] = float("inf")
    B.grad_norm(c.plan, 1.0, norm, scale, ws)
    assert np.isinf(norm.item()) and np.isnan(scale.item())


def plain_mx8(x, keep=False):
    b = x.view(-1, 32)
    e = (b.abs().amax(1).view(torch.int32) >> 23).sub(7).clamp(min=1)
    y = b * ((254 - e) << 23).view(torch.float32)[:, None]
    if keep:
        y = torch.where((b > 0) & (y < 2.0 ** -9), 2.0 ** -9, y)
    return y.to(torch.float8_e4m3fn).view(torch.uint8).view(-1), e.to(torch.uint8)


def mx8_values(codes, scale):
    return (codes.view(torch.float8_e4m3fn).float().view(-1, 32) * (scale.int() << 23).view(torch.float32)[:, None]).view(-1)


@pytest.mark.parametrize("size", [1e-14, 1e-7, 1e-3, 1.0, 1e8, 1e15, 2e18])
def test_codes_are_those_of_the_plain_evaluation(size):
    """Three steps in 8 bits leave the codes that torch's fp32 operations, each rounded by itself, leave: a tie decided the
    other way would be an eighth of the value off.  Gradients whose squares are small, ordinary and near the top."""
    n = 1 << 18
    g = torch.Generator(device="cuda").manual_seed(int(np.log10(size)) + 50)
    t = {"param": torch.zeros(n, device="cuda"), "weight_decay": 0.0}
    t |= {x: torch.zeros(n, dtype=torch.uint8, device="cuda") for x in ("m", "v")}
    t |= {x: torch.ones(n // 32, dtype=torch.uint8, device="cuda") for x in ("m_scale", "v_scale")}
    t["grad"] = torch.zeros(n, device="cuda")
    plan = B.AdamWPlan([t])
    ref = {x: t[x].clone() for x in ("m", "v", "m_scale", "v_scale")}
    scale = torch.tensor([0.7], device="cuda")
    for step in range(1, 4):
        t["grad"].copy_(torch.randn(n, generator=g, device="cuda") * size)
        x = t["grad"] * scale
        m = 0.9 * mx8_values(ref["m"], ref["m_scale"]) + (1 - 0.9) * x
        v = 0.95 * mx8_values(ref["v"], ref["v_scale"]).square() + (1 - 0.95) * x * x
        ref["m"], ref["m_scale"] = plain_mx8(m)
        ref["v"], ref["v_scale"] = plain_mx8(v.sqrt(), keep=True)
        B.adamw_step(plan, 1e-3, 0.9, 0.95, 1e-8, step, grad_scale=scale)
        for k, want in ref.items():
            assert torch.equal(t[k], want), k


def test_mx8_codes_stand_for_their_values():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    scales = torch.tensor([1, 100, 120, 127, 130, 150, 200, 240], dtype=torch.uint8, device="cuda")
    for dt in (torch.float32, torch.bfloat16):
        out = torch.empty(256, dtype=dt, device="cuda")
        B.mx8_decode(codes, scales, out)
        ref = codes.view(torch.float8_e4m3fn).double() * torch.exp2(scales.double() - 127).repeat_interleave(32)
        # bf16 keeps 2^-133 and up: the smallest scale's smallest codes are rounded there
        fine = torch.isfinite(ref) & ((ref == 0) | (ref.abs() >= 2.0 ** -126))
        assert torch.equal(out.double()[fine], ref[fine]) and bool(torch.isnan(out[torch.isnan(ref)]).all())


@pytest.mark.parametrize("n", [1, 31, 32, 33, 5000])
def test_mx8_round_trip(n):
    x = torch.randn(n, device="cuda") * torch.logspace(-6, 3, n, device="cuda")
    codes, scales = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty((n + 31) // 32, dtype=torch.uint8, device="cuda")
    out, again = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    B.mx8_encode(x, codes, scales)
    B.mx8_decode(codes, scales, out)
    ref = x.double().cpu().numpy()
    assert (np.abs(out.double().cpu().numpy() - ref) <= np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * block_scale(ref))).all()
    B.mx8_encode(out, codes, scales)
    B.mx8_decode(codes, scales, again)
    # what is held is held again as it is, unless the block's largest value was rounded up to the next power of two
    top = torch.cat([out.abs(), torch.zeros(-n % 32, device="cuda")]).view(-1, 32).amax(1)
    same = torch.frexp(top)[1] == torch.frexp(torch.cat([x.abs(), torch.zeros(-n % 32, device="cuda")]).view(-1, 32).amax(1))[1]
    keep = same.repeat_interleave(32)[:n]
    assert torch.equal(again[keep], out[keep])
