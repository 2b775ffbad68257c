"""The operators together, as one step of a layer with windowed attention and biased projections uses them: products with
bias, activation and residual, windowed attention with sinks, their gradients with the grouped products, the clipped AdamW
step on the gradients.  Forward and gradients against torch autograd in 64 bits on the same bf16 weights; the bound is the
one of this library's bf16 layers (relative Frobenius error 2e-2 per tensor)."""
import numpy as np
import pytest
import torch

from oracle import streambp_oracle as O
from paper_2506_03077_b200 import binding as B
from paper_2506_03077_b200 import dp
from helpers import TOL

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


class Block:
    """x -> q, k, v (bias) -> windowed attention -> out (bias, + x) = r -> up (bias, GELU) -> down (bias, + r) = y"""

    def __init__(self, T, d, Hq, Hkv, dh, ff, window, sinks, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(BF)
        self.T, self.d, self.Hq, self.Hkv, self.dh, self.ff, self.window, self.sinks = T, d, Hq, Hkv, dh, ff, window, sinks
        w, b = d ** -0.5, 0.1
        self.W = {"wq": rand(Hq * dh, d, std=w), "bq": rand(Hq * dh, std=b), "wk": rand(Hkv * dh, d, std=w), "bk": rand(Hkv * dh, std=b),
                  "wv": rand(Hkv * dh, d, std=w), "bv": rand(Hkv * dh, std=b), "wo": rand(d, Hq * dh, std=(Hq * dh) ** -0.5),
                  "bo": rand(d, std=b), "w1": rand(ff, d, std=w), "b1": rand(ff, std=b), "w2": rand(d, ff, std=ff ** -0.5), "b2": rand(d, std=b)}
        self.x, self.dy = rand(T, d), rand(T, d)

    def forward(self):
        T, W = self.T, self.W
        new = lambda *s: torch.empty(*s, dtype=BF, device="cuda")
        s = {"q": new(T, self.Hq, self.dh), "k": new(T, self.Hkv, self.dh), "v": new(T, self.Hkv, self.dh), "o": new(T, self.Hq, self.dh),
             "lse": torch.empty(self.Hq, T, device="cuda"), "r": new(T, self.d), "z": new(T, self.ff), "h": new(T, self.ff), "y": new(T, self.d)}
        for n in "qkv":
            B.gemm_epilogue(self.x, W["w" + n], s[n].view(T, -1), bias=W["b" + n])
        B.attention_window_forward(s["q"], s["k"], s["v"], 0, self.window, self.sinks, s["o"], s["lse"])
        B.gemm_epilogue(s["o"].view(T, -1), W["wo"], s["r"], bias=W["bo"], residual=self.x)
        B.gemm_epilogue(s["r"], W["w1"], s["h"], bias=W["b1"], activation="gelu_tanh", pre=s["z"])
        B.gemm_epilogue(s["h"], W["w2"], s["y"], bias=W["b2"], residual=s["r"])
        return s

    def backward(self, s, grads):
        """grads: fp32 views (overwritten).  Returns dx."""
        T = self.T
        new = lambda *sh: torch.empty(*sh, dtype=BF, device="cuda")
        ws = lambda N: B.alloc_workspace(B.gemm_epilogue_workspace_bytes(T, N))
        W = self.W
        # down: dy is dz of the last product and the residual's gradient
        B.gemm_epilogue_backward(self.dy, None, "none", None, grads["b2"], ws(self.d))
        dh = new(T, self.ff)
        B.gemm_grouped([(B.OP_NN, [(self.dy, W["w2"])], dh, False), (B.OP_TN, [(self.dy, s["h"])], grads["w2"], False)])
        dz = new(T, self.ff)
        B.gemm_epilogue_backward(dh, s["z"], "gelu_tanh", dz, grads["b1"], ws(self.ff))
        dr = new(T, self.d)
        B.gemm_grouped([(B.OP_TN, [(dz, s["r"])], grads["w1"], False)])
        eye = torch.eye(self.d, dtype=BF, device="cuda")
        B.gemm_grouped([(B.OP_NN, [(dz, W["w1"]), (self.dy, eye)], dr, False)])        # + the residual's gradient
        # out
        B.gemm_epilogue_backward(dr, None, "none", None, grads["bo"], ws(self.d))
        do = new(T, self.Hq, self.dh)
        B.gemm_grouped([(B.OP_NN, [(dr, W["wo"])], do.view(T, -1), False), (B.OP_TN, [(dr, s["o"].view(T, -1))], grads["wo"], False)])
        g = {n: torch.empty_like(s[n]) for n in "qkv"}
        aws = B.alloc_workspace(B.attention_window_workspace_bytes(T, 0, self.Hq, self.Hkv, self.dh, self.window, self.sinks))
        B.attention_window_backward(s["q"], s["k"], s["v"], s["o"], do, s["lse"], 0, self.window, self.sinks, g["q"], g["k"], g["v"], aws)
        flat = {n: g[n].view(T, -1) for n in "qkv"}
        for n in "qkv":
            B.gemm_epilogue_backward(flat[n], None, "none", None, grads["b" + n], ws(flat[n].shape[1]))
        dx = new(T, self.d)
        B.gemm_grouped([(B.OP_TN, [(flat[n], self.x)], grads["w" + n], False) for n in "qkv"])
        B.gemm_grouped([(B.OP_NN, [(flat[n], W["w" + n]) for n in "qkv"], dx, False)])
        dx2 = new(T, self.d)
        B.gemm_epilogue(dx, eye, dx2, residual=dr)
        return dx2

    def reference(self):
        """y, dx, all parameter gradients and dk by autograd in 64 bits."""
        P = {k: v.double().requires_grad_() for k, v in self.W.items()}
        x = self.x.double().requires_grad_()
        T, G = self.T, self.Hq // self.Hkv
        q, k, v = ((x @ P["w" + n].T + P["b" + n]).view(T, -1, self.dh) for n in "qkv")
        k.retain_grad()
        t = torch.arange(T, device="cuda")
        see = (t[None] <= t[:, None]) & ((t[:, None] - t[None] < self.window) | (t[None] < self.sinks))
        a = torch.einsum("thd,jhd->htj", q, k.repeat_interleave(G, 1)) * self.dh ** -0.5
        o = torch.einsum("htj,jhd->thd", a.masked_fill(~see, -torch.inf).softmax(-1), v.repeat_interleave(G, 1))
        r = o.reshape(T, -1) @ P["wo"].T + P["bo"] + x
        y = torch.nn.functional.gelu(r @ P["w1"].T + P["b1"], approximate="tanh") @ P["w2"].T + P["b2"] + r
        y.backward(self.dy.double())
        return y.detach(), x.grad, {n: p.grad for n, p in P.items()}, k.grad


def shapes_of(block):
    return {k: tuple(v.shape) for k, v in block.W.items()}


@pytest.mark.parametrize("T,d,Hq,Hkv,dh,ff,window,sinks", [(300, 256, 4, 2, 64, 688, 70, 3), (515, 512, 4, 1, 128, 1024, 200, 0)])
def test_block_forward_backward_and_step(T, d, Hq, Hkv, dh, ff, window, sinks):
    blk = Block(T, d, Hq, Hkv, dh, ff, window, sinks)
    bucket = dp.GradBucket(shapes_of(blk), 1)
    params = dp.ParamBucket(bucket, blk.W)
    blk.W = params.views                               # the products read the buffer that the step writes
    bucket.flat.fill_(float("nan"))                    # every gradient is overwritten; what lies between takes no part
    s = blk.forward()
    dx = blk.backward(s, bucket.views)
    y, dx_ref, g_ref, dk_ref = blk.reference()
    rel = lambda a, b: O.rel_frobenius(a.double().cpu().numpy(), b.double().cpu().numpy())
    assert rel(s["y"], y) <= TOL[BF] and rel(dx, dx_ref) <= TOL[BF]
    # A key bias adds the same number to all scores of a row, which the softmax does not see: its gradient, the sum over the
    # rows of dk, is zero, and there is nothing that an error could be relative to.  What the sum carries is the errors e_j
    # of the rows of dk: |sum_j e_j| <= sqrt(T) |e|_F (Cauchy-Schwarz), and |e|_F <= TOL |dk|_F is the bound of that tensor.
    assert float(g_ref["bk"].norm()) <= 1e-10 * float(dk_ref.norm())
    assert float(bucket.views["bk"].double().norm()) <= T ** 0.5 * TOL[BF] * float(dk_ref.norm())
    for k in g_ref.keys() - {"bk"}:
        assert rel(bucket.views[k], g_ref[k]) <= TOL[BF], k

    # one clipped step on these gradients, 8-bit moments from zero: m = 0.1 g s, the root of v exactly |g s| sqrt(0.05)
    before = {k: v.double() for k, v in blk.W.items()}
    decay = {k: 0.1 for k in g_ref if k.startswith("w")}
    opt = dp.ShardedAdamW(params, bucket, bucket.flat, decay, bits=8)
    opt.step(lr=1e-2, max_norm=0.5)
    norm = float(torch.sqrt(sum((v.double() ** 2).sum() for v in bucket.views.values())))
    assert abs(opt.norm.item() - norm) <= 1e-6 * norm
    scale = min(1.0, 0.5 / (norm + 1e-6))
    for k, v in blk.W.items():
        # the step of a first update is lr times the sign, up to eps; the parameter is the fp32 master rounded once
        g = bucket.views[k].double() * scale
        want = before[k] * (1 - 1e-2 * decay.get(k, 0.0)) - 1e-2 * g / (g.abs() + 1e-8)
        assert bool(((v.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all()), k
    # and the next forward runs on the new parameters
    s2 = blk.forward()
    assert bool(torch.isfinite(s2["y"]).all()) and not torch.equal(s["y"], s2["y"])


class OtherRank:
    """torch.distributed as rank `rank` of two sees it, the other rank's numbers known beforehand (both run in this process,
    one after the other)."""

    def __init__(self, others_square):
        self.others_square, self.gathered = others_square, None

    def is_initialized(self):
        return False

    def get_backend(self, group=None):
        return "none"

    def all_reduce(self, t, group=None):
        t += self.others_square

    def all_gather(self, parts, x, group=None):
        for p in parts:
            p.copy_(x)
        self.gathered = x.clone()


@pytest.mark.parametrize("bits", [8, 32])
def test_two_shards_step_as_one(monkeypatch, bits):
    shapes = {"a": (100, 70), "b": (333,), "c": (64, 128), "d": (5,)}
    g = torch.Generator(device="cuda").manual_seed(0)
    values = {k: (torch.randn(s, generator=g, device="cuda") * 0.02).to(BF) for k, s in shapes.items()}
    decay = {"a": 0.1, "c": 0.1}
    one, two = dp.GradBucket(shapes, 1), dp.GradBucket(shapes, 2)
    for k in shapes:
        x = torch.randn(shapes[k], generator=g, device="cuda") * 1e-3
        one.views[k].copy_(x)
        two.views[k].copy_(x)
    p1 = dp.ParamBucket(one, values)
    whole = dp.ShardedAdamW(p1, one, one.flat, decay, bits=bits)
    ranks = []
    for r in range(2):
        lo, hi = two.shard_range(r)
        ranks.append((dp.ParamBucket(two, values), two.flat[lo:hi].clone()))
    opts = [dp.ShardedAdamW(p, two, s, decay, bits=bits, rank=r, world=2) for r, (p, s) in enumerate(ranks)]
    for _ in range(3):
        whole.step(lr=1e-2, max_norm=0.01)
        for r, opt in enumerate(opts):
            fake = OtherRank((ranks[1 - r][1].double() ** 2).sum())
            monkeypatch.setattr(dp, "dist", fake)
            opt.step(lr=1e-2, max_norm=0.01)
            monkeypatch.undo()
            lo, hi = two.shard_range(r)
            ranks[r][0].flat[lo:hi].copy_(fake.gathered)      # its own slice, as the gather of both would leave it
    for k in shapes:
        o, n = two.table[k]
        got = torch.cat([ranks[0][0].flat[:two.shard_elems], ranks[1][0].flat[two.shard_elems:]])[o:o + n].view(shapes[k])
        # the clip factor of the two sides differs by an fp32 rounding or two; blocks of moments are the same
        assert torch.allclose(got.float(), p1.views[k].float(), rtol=2.0 ** -7, atol=1e-6), k


def test_layer_backward_then_sharded_step():
    """streambp_layer_backward through the data-parallel wrapper, then its shard through the optimizer."""
    from paper_2506_03077_b200 import synth
    shape = synth.LayerShape(256, 4, 2, 64, 688, True, 1e4)
    W = {k: torch.from_numpy(v).cuda().to(BF) for k, v in synth.make_layer_weights(shape, 3, True).items()}
    cfg = B.LayerConfig(256, 4, 2, 64, 688, True, 1e4, 1e-6, BF)
    X, dY = (torch.from_numpy(a).cuda().to(BF) for a in synth.make_layer_io(shape, 4, 200, True))
    bucket = dp.GradBucket(B.layer_grad_shapes(cfg), 1)
    params = dp.ParamBucket(bucket, W)
    r = dp.DataParallelLayerBackward(cfg, params.views, 200, 64)
    opt = dp.ShardedAdamW(params, r.bucket, r.shard, {k: 0.1 for k in W if k.startswith("w")}, bits=8)
    dX = torch.empty_like(X)
    losses = []
    for _ in range(3):
        r.step(X, dY, dX)
        r.wait()
        before, master = params.flat.clone(), opt.master.clone()
        opt.step(lr=1e-3)
        # seen in the master copy: a gain of one, in steps of 2^-8 or 2^-7 in bf16, need not leave its value for a step of
        # 1e-3, less than half of either
        changed = {k: not torch.equal(master[o:o + n], opt.master[o:o + n]) for k, (o, n) in bucket.table.items()}
        assert all(changed.values())
        pad = torch.ones_like(before, dtype=torch.bool)
        for o, n in bucket.table.values():
            pad[o:o + n] = False
        assert torch.equal(before[pad], params.flat[pad])
        losses.append(opt.norm.item())
    assert np.isfinite(losses).all() and bool(torch.isfinite(params.flat).all())
