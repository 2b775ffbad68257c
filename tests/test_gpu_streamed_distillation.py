"""A teacher's lists into a student's streamed head, layer norm and table behind it: scoring chunk by chunk, embedding, layer norm, the
streamed distilling head (which norms its input itself), and the gradients back to the table, against autograd in 64 bits."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from helpers import TOL
from test_gpu_logprobs import BF, F32
from test_gpu_model_ends import relative

pytestmark = pytest.mark.gpu


class Student:
    def __init__(self, dtype=BF, T=200, V=2003, d=256, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=g, device="cuda") * std + mean).to(dtype)
        new = lambda *s, t=dtype: torch.empty(*s, dtype=t, device="cuda")
        self.T, self.V, self.d, self.dtype, self.scale, self.chunk = T, V, d, dtype, math.sqrt(d), 64
        self.P = {"table": rand(V, d, std=d ** -0.5), "gain": rand(d, std=0.1, mean=1.0), "bias": rand(d, std=0.1),
                  "g_final": rand(d, std=0.1, mean=1.0), "out": rand(V, d, std=2 * d ** -0.5)}
        self.teacher = {"H": rand(T, d), "out": rand(V, d, std=3 * d ** -0.5)}
        self.ids = torch.randint(V // 8, (T,), generator=g, device="cuda")
        self.weight = torch.full((T,), 1.0 / T, device="cuda")
        self.weight[:70] = 0
        self.cfg = B.HeadConfig(d, V, dtype=dtype)
        self.G = {n: new(*p.shape, t=F32) for n, p in self.P.items()}
        self.b = {n: new(T, d) for n in ("x", "h", "dh", "dx")} | {n: new(T, t=F32) for n in ("mean", "rstd", "row")}
        self.b |= {"loss": new(1, t=F32), "list": new(T, 12, t=torch.int64), "values": new(T, 12, t=F32)}
        self.ws = {"score": B.lmhead_logprobs_workspace_bytes(self.cfg, T, self.chunk), "embed": B.embedding_workspace_bytes(),
                   "head": B.lmhead_distill_workspace_bytes(self.cfg, T, self.chunk, 2), "norm": B.layernorm_workspace_bytes(T, d),
                   "table": B.embedding_backward_workspace_bytes(T, V, d)}
        self.ws = {n: B.alloc_workspace(size) for n, size in self.ws.items()}

    def run(self):
        P, G, b, w = self.P, self.G, self.b, self.ws
        B.lmhead_logprobs(self.cfg, P["g_final"], self.teacher["out"], self.teacher["H"], None, self.chunk, w["score"], top_logp=b["values"], top_ids=b["list"])
        B.embedding_forward(P["table"], self.ids, b["x"], w["embed"], scale=self.scale)
        B.layernorm_forward(b["x"], P["gain"], P["bias"], 1e-5, b["h"], b["mean"], b["rstd"])
        B.lmhead_distill_backward(self.cfg, P["g_final"], P["out"], b["h"], b["list"], b["values"], self.weight, self.chunk, b["loss"], b["dh"], G["out"],
                                  G["g_final"], w["head"], row_loss=b["row"], tail=True, wgrad_group=2)
        B.layernorm_backward(b["dh"], b["x"], P["gain"], b["mean"], b["rstd"], dx=b["dx"], d_gain=G["gain"], d_bias=G["bias"], workspace=w["norm"])
        B.embedding_backward(b["dx"], self.ids, G["table"], w["table"], scale=self.scale)

    def results(self):
        return {n: t.clone() for n, t in self.G.items()} | {n: self.b[n].clone() for n in ("loss", "row", "list")}

    def reference(self):
        P = {n: p.double().requires_grad_() for n, p in self.P.items()}
        h = torch.nn.functional.layer_norm(P["table"][self.ids] * self.scale, (self.d,), P["gain"], P["bias"], 1e-5)
        hn = h * torch.rsqrt((h * h).mean(1, keepdim=True) + self.cfg.rms_eps) * P["g_final"]
        lp = torch.log_softmax(hn @ P["out"].T, 1)
        q, c = self.b["values"].double().exp(), self.b["list"]
        rest, listed = 1 - q.sum(1), lp.gather(1, c)
        row = (q * (q.log() - listed)).sum(1) + rest * (rest.log() - torch.logsumexp(lp.scatter(1, c, -math.inf), 1))
        row = torch.where(self.weight != 0, row, 0.0)
        loss = (row * self.weight.double()).sum()
        return loss.detach(), row.detach(), dict(zip(P, torch.autograd.grad(loss, list(P.values()))))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_step(dtype):
    s = Student(dtype)
    s.run()
    got = s.results()
    loss, row, grads = s.reference()
    assert abs(got["loss"].item() - loss.item()) <= TOL[dtype] * abs(loss.item()) and relative(got["row"], row) <= TOL[dtype]
    for n, ref in grads.items():
        assert relative(got[n], ref) <= TOL[dtype], n
    assert all(B.last_device_status(w) == B.OK for w in s.ws.values())


def test_steps_at_once_and_replayed():
    """two students on streams of their own, captured and replayed with other inputs"""
    a, b = Student(seed=1), Student(seed=2)
    for s in (a, b):
        s.run()
    want = [s.results() for s in (a, b)]
    graphs, streams = [torch.cuda.CUDAGraph() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for s, graph, stream in zip((a, b), graphs, streams):
        with torch.cuda.graph(graph, stream=stream):
            s.run()
    for change in (False, True):
        if change:                          # each takes the other's parameters
            for p, q in [(a.P[n], b.P[n]) for n in a.P] + [(a.teacher[n], b.teacher[n]) for n in a.teacher] + [(a.ids, b.ids)]:
                keep = p.clone()
                p.copy_(q)
                q.copy_(keep)
            want.reverse()
        for s in (a, b):
            for g in s.G.values():
                g.fill_(5.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s, w in zip((a, b), want):
            got = s.results()
            assert all(torch.equal(got[n], w[n]) for n in w)
