"""The operators of a model's two ends together: the streamed heads against the operators on whole logits, a training step of
embedding, norms and a distilled head against autograd in 64 bits, calls at once, on other streams and replayed from graphs."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from paper_2506_03077_b200 import synth
from helpers import TOL, to_dev
from test_gpu_distill import teacher
from test_gpu_logprobs import BF, F32

pytestmark = pytest.mark.gpu


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


class Head:
    def __init__(self, dtype, T=200, d=256, V=2003, seed=0):
        bf = dtype == BF
        g, W, H, labels = synth.make_head_inputs(synth.HeadShape(d, V), seed, T, bf, T // 4)
        self.cfg = B.HeadConfig(d, V, dtype=dtype)
        self.g, self.W, self.H = (to_dev(x, dtype) for x in (g, W, H))
        self.W *= 8                                   # (logits that tell tokens apart)
        self.labels, self.T, self.V, self.d, self.dtype = torch.from_numpy(labels).cuda(), T, V, d, dtype

    def logits(self, H=None, g=None, W=None):
        """in 64 bits, the norm's output rounded as the library stores it (straight through for gradients)"""
        H, g, W = (a if a is not None else b.double() for a, b in ((H, self.H), (g, self.g), (W, self.W)))
        h = H * torch.rsqrt((H * H).mean(1, keepdim=True) + self.cfg.rms_eps) * g
        return (h + (h.detach().to(self.dtype).double() - h.detach())) @ W.T

    def score(self, tokens, chunk, k, tau=1.0, status=B.OK):
        out = {x: torch.full((self.T,), 7.0, device="cuda") for x in ("logp", "lse", "entropy")}
        out["top_logp"], out["top_ids"] = torch.full((self.T, k), 7.0, device="cuda"), torch.full((self.T, k), 7, device="cuda")
        if tokens is None:
            out["logp"] = None
        ws = B.alloc_workspace(B.lmhead_logprobs_workspace_bytes(self.cfg, self.T, chunk))
        B.lmhead_logprobs(self.cfg, self.g, self.W, self.H, tokens, chunk, ws, temperature=tau, **out)
        assert B.last_device_status(ws) == status
        return out

    def distill(self, ids, values, w, chunk, group=1, accumulate=False, start=7.0, status=B.OK, **kw):
        loss, row = torch.full((1,), 7.0, device="cuda"), torch.full((self.T,), 7.0, device="cuda")
        dH, dW = torch.full_like(self.H, 7.0), torch.full((self.V, self.d), start, device="cuda")
        dg = torch.full((self.d,), start, device="cuda")
        ws = B.alloc_workspace(B.lmhead_distill_workspace_bytes(self.cfg, self.T, chunk, group))
        B.lmhead_distill_backward(self.cfg, self.g, self.W, self.H, ids, values, w, chunk, loss, dH, dW, dg, ws, row_loss=row,
                                  accumulate=accumulate, wgrad_group=group, **kw)
        assert B.last_device_status(ws) == status
        return loss, row, dH, dW, dg


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("chunk", [64, 48, 1000])
def test_scoring_head(dtype, chunk):
    h = Head(dtype)
    got = h.score(h.labels, chunk, 10, 0.7)
    lp = torch.log_softmax(h.logits() / 0.7, 1)
    part = h.labels != -100
    want = torch.where(part, lp.gather(1, torch.where(part, h.labels, 0)[:, None])[:, 0], 0.0)
    # logits of 8 sqrt(256) 0.02 = 2.6 summed in fp32 over exact products; a norm's output that sits at a border of bf16 may
    # be rounded the other way: one of 256 operands off by 2^-8 of itself
    tol = 1e-4 if dtype == F32 else 2e-2
    assert ((got["logp"].double() - want).abs() <= tol).all() and (got["logp"][~part] == 0).all()
    assert (got["top_ids"][~part] == -1).all() and (got["top_logp"][~part] == -math.inf).all()
    listed = got["top_ids"][part]
    assert ((got["top_logp"][part].double() - lp[part].gather(1, listed)).abs() <= tol).all()
    assert ((lp[part].sort(1, descending=True).values[:, :10] - got["top_logp"][part]).abs() <= tol).all()
    # without tokens every row is scored; the same bits
    free = h.score(None, chunk, 10, 0.7)
    assert all(torch.equal(free[x][part], got[x][part]) for x in ("lse", "entropy", "top_logp", "top_ids"))
    assert ((free["entropy"].double() + (lp.exp() * lp).sum(1)).abs() <= 10 * tol).all()


def test_scoring_head_agrees_with_the_objectives():
    """logp as the GRPO head reports it"""
    h = Head(BF)
    got = h.score(h.labels, 64, 4)["logp"]
    z = torch.zeros(h.T, device="cuda")
    logp = torch.empty(h.T, device="cuda")
    loss, dH, dW, dg = torch.empty(1, device="cuda"), torch.empty_like(h.H), torch.empty(h.V, h.d, device="cuda"), torch.empty(h.d, device="cuda")
    ws = B.alloc_workspace(B.lmhead_workspace_bytes(h.cfg, h.T, 64))
    B.lmhead_rl_backward(h.cfg, B.OBJ_GRPO, 0.0, 0.2, h.g, h.W, h.H, h.labels, z, z, z, z, 64, loss, dH, dW, dg, ws, logp=logp)
    assert ((got - logp).abs() <= 3e-5 + 2.0 ** -22 * logp.abs()).all()


def test_scoring_head_with_bad_tokens():
    h = Head(BF)
    t = h.labels.clone()
    t[100] = h.V
    got = h.score(t, 64, 3, status=B.E_BAD_LABEL)
    assert got["logp"][100] == 0 and (got["top_ids"][100] == -1).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("chunk,group,tail", [(64, 1, False), (48, 3, True), (1000, 1, True), (32, 2, False)])
def test_distilling_head(dtype, chunk, group, tail):
    h = Head(dtype)
    tau = 2.0
    ids, values = teacher(h.logits(), 12, tau, tail)
    w = torch.where(h.labels != -100, 1.0 / h.T, 0.0).float()
    w[120:128] = 0
    loss, row, dH, dW, dg = h.distill(ids, values, w, chunk, group, temperature=tau, tail=tail)
    H, g, W = (x.double().requires_grad_() for x in (h.H, h.g, h.W))
    lp = torch.log_softmax(h.logits(H, g, W) / tau, 1)
    q = values.double().exp() if tail else torch.softmax(values.double() / tau, 1)
    want = (q * (q.log() - lp.gather(1, ids))).sum(1)
    if tail:
        r = 1 - q.sum(1)
        want = want + r * (r.log() - torch.log1p(-lp.gather(1, ids).exp().sum(1)))
    want = torch.where(w != 0, want, 0.0)
    total = (want * w.double()).sum()
    grads = torch.autograd.grad(total, (H, g, W))
    assert abs(loss.item() - total.item()) <= (1e-4 if dtype == F32 else 2e-2) * abs(total.item())
    assert (row[w == 0] == 0).all() and (dH[w == 0] == 0).all()
    for got, ref in zip((dH, dg, dW), grads):
        assert relative(got, ref) <= TOL[dtype]
    more = h.distill(ids, values, w, chunk, group, True, 0.25, temperature=tau, tail=tail)
    assert torch.equal(more[2], dH) and relative(more[3] - 0.25, dW.double()) <= 1e-3 and torch.equal(more[0], loss)


def test_distilling_head_without_rows():
    h = Head(BF)
    ids, values = teacher(h.logits(), 4, 1.0, False)
    loss, row, dH, dW, dg = h.distill(ids, values, torch.zeros(h.T, device="cuda"), 64, status=B.E_NO_VALID_LABELS)
    assert loss.item() == 0 and all((x == 0).all() for x in (row, dH, dW, dg))
    ids[150, 1] = h.V
    h.distill(ids, values, torch.ones(h.T, device="cuda"), 64, status=B.E_BAD_LABEL)


class Step:
    """table[ids] sqrt(d) -> layer norm -> up with GELU -> down + its input -> layer norm -> logits -> distillation from a
    teacher's list, and the gradients of all of it"""

    def __init__(self, T=300, V=3001, d=256, ff=512, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=g, device="cuda") * std + mean).to(BF)
        self.T, self.V, self.d, self.ff, self.scale = T, V, d, ff, math.sqrt(d)
        self.P = {"table": rand(V, d, std=1 / math.sqrt(d)), "g1": rand(d, std=0.1, mean=1.0), "b1": rand(d, std=0.1), "w1": rand(ff, d, std=d ** -0.5),
                  "c1": rand(ff, std=0.1), "w2": rand(d, ff, std=ff ** -0.5), "c2": rand(d, std=0.1), "g2": rand(d, std=0.1, mean=1.0),
                  "b2": rand(d, std=0.1), "out": rand(V, d, std=2 * d ** -0.5)}
        self.ids = torch.randint(V // 4, (T,), generator=g, device="cuda")
        self.ids[5:25] = 11
        self.teacher_H = rand(T, d)
        self.cfg = B.HeadConfig(d, V, dtype=BF)
        new = lambda *s, t=BF: torch.empty(*s, dtype=t, device="cuda")
        self.b = {n: new(T, d) for n in ("x", "h1", "r", "h2", "dh2", "dr", "dh1", "dx")}
        self.b |= {n: new(T, ff) for n in ("a", "z", "da", "dz")}
        self.b |= {"logits": new(T, V), "dlogits": new(T, V), "row": new(T, t=F32), "ids": new(T, 16, t=torch.int64), "values": new(T, 16, t=F32)}
        for n in ("m1", "s1", "m2", "s2"):
            self.b[n] = new(T, t=F32)
        self.G = {n: new(*p.shape, t=F32) for n, p in self.P.items()}
        self.weight = torch.full((T,), 1.0 / T, device="cuda")
        self.weight[:40] = 0
        ws = lambda n: B.alloc_workspace(n)
        self.ws = {"embed": ws(B.embedding_workspace_bytes()), "dembed": ws(B.embedding_backward_workspace_bytes(T, V, d)),
                   "norm": ws(B.layernorm_workspace_bytes(T, d)), "distill": ws(B.distill_topk_workspace_bytes()),
                   "ff": ws(B.gemm_epilogue_workspace_bytes(T, ff)), "d": ws(B.gemm_epilogue_workspace_bytes(T, d)),
                   "score": ws(B.lmhead_logprobs_workspace_bytes(self.cfg, T, 128))}

    def run(self, stream=None):
        P, b, G, w, kw = self.P, self.b, self.G, self.ws, {"stream": stream}
        B.lmhead_logprobs(self.cfg, P["g2"], P["out"], self.teacher_H, None, 128, w["score"], top_logp=b["values"], top_ids=b["ids"], **kw)
        B.embedding_forward(P["table"], self.ids, b["x"], w["embed"], scale=self.scale, **kw)
        B.layernorm_forward(b["x"], P["g1"], P["b1"], 1e-5, b["h1"], b["m1"], b["s1"], **kw)
        B.gemm_epilogue(b["h1"], P["w1"], b["a"], bias=P["c1"], activation="gelu", pre=b["z"], **kw)
        B.gemm_epilogue(b["a"], P["w2"], b["r"], bias=P["c2"], residual=b["x"], **kw)
        B.layernorm_forward(b["r"], P["g2"], P["b2"], 1e-5, b["h2"], b["m2"], b["s2"], **kw)
        B.gemm_epilogue(b["h2"], P["out"], b["logits"], **kw)
        B.distill_topk(b["logits"], b["ids"], b["values"], b["row"], w["distill"], d_logits=b["dlogits"], weight=self.weight, tail=True, **kw)
        B.gemm(B.OP_NN, b["dlogits"], P["out"], b["dh2"], **kw)
        B.gemm(B.OP_TN, b["dlogits"], b["h2"], G["out"], **kw)
        B.layernorm_backward(b["dh2"], b["r"], P["g2"], b["m2"], b["s2"], dx=b["dr"], d_gain=G["g2"], d_bias=G["b2"], workspace=w["norm"], **kw)
        B.gemm_epilogue_backward(b["dr"], None, "none", None, G["c2"], w["d"], **kw)
        B.gemm_grouped([(B.OP_NN, [(b["dr"], P["w2"])], b["da"], False), (B.OP_TN, [(b["dr"], b["a"])], G["w2"], False)], **kw)
        B.gemm_epilogue_backward(b["da"], b["z"], "gelu", b["dz"], G["c1"], w["ff"], **kw)
        B.gemm_grouped([(B.OP_NN, [(b["dz"], P["w1"])], b["dh1"], False), (B.OP_TN, [(b["dz"], b["h1"])], G["w1"], False)], **kw)
        B.layernorm_backward(b["dh1"], b["x"], P["g1"], b["m1"], b["s1"], dx=b["dx"], d_gain=G["g1"], d_bias=G["b1"], add=b["dr"],
                             workspace=w["norm"], **kw)
        B.embedding_backward(b["dx"], self.ids, G["table"], w["dembed"], scale=self.scale, **kw)

    def results(self):
        return {n: t.clone() for n, t in self.G.items()} | {"row": self.b["row"].clone(), "ids": self.b["ids"].clone()}

    def reference(self):
        P = {n: p.double().requires_grad_() for n, p in self.P.items()}
        F = torch.nn.functional
        x = P["table"][self.ids] * self.scale
        h = F.layer_norm(x, (self.d,), P["g1"], P["b1"], 1e-5)
        r = F.gelu(h @ P["w1"].T + P["c1"]) @ P["w2"].T + P["c2"] + x
        lp = torch.log_softmax(F.layer_norm(r, (self.d,), P["g2"], P["b2"], 1e-5) @ P["out"].T, 1)
        q = self.b["values"].double().exp()
        rest = 1 - q.sum(1)
        row = (q * (q.log() - lp.gather(1, self.b["ids"]))).sum(1) + rest * (rest.log() - torch.log1p(-lp.gather(1, self.b["ids"]).exp().sum(1)))
        return row.detach(), dict(zip(P, torch.autograd.grad((row * self.weight.double()).sum(), list(P.values()))))


def test_a_training_step():
    s = Step()
    s.run()
    got = s.results()
    row, grads = s.reference()
    on = s.weight != 0
    assert relative(got["row"][on], row[on]) <= TOL[BF] and (got["row"][~on] == 0).all()
    for n, ref in grads.items():
        assert relative(got[n], ref) <= TOL[BF], (n, relative(got[n], ref))
    s.run()
    again = s.results()
    assert all(torch.equal(again[n], got[n]) for n in got)


def test_a_training_step_replayed_and_on_other_streams():
    s, t = Step(), Step(seed=9)
    s.run()
    t.run()
    want_s, want_t = s.results(), t.results()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for st in (a, b):
        st.wait_stream(torch.cuda.current_stream())
    for x in (s, t):
        for g in x.G.values():
            g.fill_(5.0)
    torch.cuda.synchronize()
    s.run(a)                        # two steps at once
    t.run(b)
    torch.cuda.synchronize()
    for x, want in ((s, want_s), (t, want_t)):
        got = x.results()
        assert all(torch.equal(got[n], want[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    s.ids.copy_(t.ids)
    for n in s.P:
        s.P[n].copy_(t.P[n])
    s.teacher_H.copy_(t.teacher_H)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    got = s.results()
    assert all(torch.equal(got[n], want_t[n]) for n in want_t)
    assert B.last_device_status(s.ws["dembed"]) == B.OK and B.last_device_status(s.ws["distill"]) == B.OK


def test_refused_tensors():
    z = torch.zeros(4, 100, device="cuda")
    ws = B.alloc_workspace(4096)
    ids, values = torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(4, 3, device="cuda")
    row = torch.zeros(4, device="cuda")
    bad = [lambda: B.token_logprobs(z, ids[:, 0].clone().int(), ws, lse=row), lambda: B.token_logprobs(z, None, ws, lse=row[:3].clone()),
           lambda: B.token_logprobs(z.cpu(), None, ws, lse=row), lambda: B.token_logprobs(z.t(), None, ws, lse=row),
           lambda: B.token_logprobs(z, None, ws.cpu(), lse=row), lambda: B.token_logprobs(z, None, ws, lse=row, top_ids=ids, top_logp=values[:, :2].clone()),
           lambda: B.distill_topk(z, ids, values[:, :2].contiguous(), row, ws), lambda: B.distill_topk(z, ids, values, row.double(), ws),
           lambda: B.distill_topk(z, ids, values, row, ws, d_logits=z.bfloat16()), lambda: B.layernorm_forward(z, row, None, 1e-5, z),
           lambda: B.layernorm_forward(z, None, None, 1e-5, z.bfloat16()), lambda: B.embedding_forward(z, ids.int(), z, ws),
           lambda: B.embedding_backward(z, torch.zeros(4, dtype=torch.int64, device="cuda"), z[:, :50].contiguous(), ws),
           lambda: B.token_logprobs(z.half(), None, ws, lse=row)]
    for f in bad:
        with pytest.raises((ValueError, TypeError)):
            f()
