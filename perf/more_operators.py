"""What is measured of the operators at the two ends of a model: log-probabilities of given tokens with entropy and the
top alternatives (and their gradient), distillation from a teacher's top logits (loss and gradient), layer norm (forward
and backward), and the embedding lookup with its gradient.

Each operator has a plain form made of elementary torch operations (`own` false) and the call a user makes of the
library (`own` true).  Cases are dicts of plain values; `listed()` names the fixed ones, `draw()` spreads over the
same ranges."""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _score(name, rows, vocab, top, dtype="f32", temperature=1.0, pad=0, masked=0, skipped=0.0):
    """`pad`: columns behind each row of a wider buffer; `masked`: last columns at minus infinity; `skipped`: share of
    rows that take no part"""
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "temperature": temperature,
            "pad": pad, "masked": masked, "skipped": skipped}


def _score_grad(name, rows, vocab, dtype="bf16", temperature=1.0, pad=0, skipped=0.0):
    return {"name": name, "op": "score_grad", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature,
            "pad": pad, "masked": 0, "skipped": skipped}


def _distill(name, rows, vocab, top, dtype="f32", temperature=1.0, tail=False, pad=0, skipped=0.0):
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "temperature": temperature,
            "tail": tail, "pad": pad, "masked": 0, "skipped": skipped}


def _norm(name, op, rows, width, dtype="bf16", add=False):
    return {"name": name, "op": op, "rows": rows, "width": width, "dtype": dtype, "add": add}


def _embed(name, op, tokens, vocab, width, dtype="bf16", accumulate=True):
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "accumulate": accumulate}


def listed():
    return [
        # a teacher's or a reference model's pass over one chunk of a streamed head: fp32 logits, 16 alternatives kept
        _score("score_chunk", 1024, 152064, 16),
        # the tokens that a sampler has just drawn, one a sequence: latency counts
        _score("score_few_rows", 3, 152064, 20, "bf16", temperature=0.7, masked=64),
        # gradient of a policy's log-probabilities with an entropy bonus, prompts left out
        _score_grad("score_grad", 2048, 32003, "bf16", skipped=0.2),
        # one chunk of a streamed head under distillation, logits overwritten by their gradient's values in fp32
        _distill("distill_chunk", 1024, 152064, 32, temperature=2.0),
        # bf16 logits of a ragged vocabulary, a long list with the rest of the teacher's mass in one bucket
        _distill("distill_tail", 1500, 50001, 100, "bf16", tail=True, skipped=0.2),
        # a few rows of a small vocabulary
        _distill("distill_few_rows", 6, 4096, 8, tail=True),
        # the norm in front of a projection, a batch of 16k rows
        _norm("norm", "norm", 16384, 4096),
        # its gradient, with the residual's gradient added and the sums of gain and bias
        _norm("norm_grad", "norm_grad", 16384, 4096, add=True),
        # the same of a ragged chunk of odd width in the precision mode
        _norm("norm_grad_ragged", "norm_grad", 1001, 1537, "f32"),
        # lookup of a long sequence, scaled by the root of the width
        _embed("embed", "embed", 32768, 152064, 3584),
        # its gradient added to what a tied head has left there; tokens as frequent as words are
        _embed("embed_grad", "embed_grad", 32768, 152064, 3584),
        # a short prompt on a small table, overwritten
        _embed("embed_grad_few", "embed_grad", 50, 4096, 256, accumulate=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in {c["op"] for c in listed()}}
    while True:
        op = rng.choice(("score", "score", "score_grad", "distill", "distill", "norm", "norm_grad", "embed", "embed_grad"))
        dtype = rng.choice(("bf16", "f32"))
        rows = _log(rng, 1, 4096)
        vocab = rng.choice((_log(rng, 200, 160000), 8 * _log(rng, 25, 20000)))
        heat, pad = rng.choice((1.0, 1.0, 0.7, 2.0)), rng.choice((0, 0, 5, 64))
        if op == "score":
            c = _score("", rows, vocab, rng.choice((0, 1, 5, 16, 20, 64, 128)), dtype, heat, pad, rng.choice((0, 0, 64)), rng.choice((0.0, 0.3)))
        elif op == "score_grad":
            c = _score_grad("", rows, vocab, dtype, heat, pad, rng.choice((0.0, 0.3)))
        elif op == "distill":
            c = _distill("", rows, vocab, rng.choice((1, 8, 20, 32, 64, 100, 128)), dtype, heat, rng.random() < 0.5, pad, rng.choice((0.0, 0.3)))
        elif op.startswith("norm"):
            c = _norm("", op, _log(rng, 1, 32768), rng.choice((_log(rng, 64, 16384), 64 * _log(rng, 1, 256))), dtype, op == "norm_grad" and rng.random() < 0.5)
        else:
            c = _embed("", op, _log(rng, 1, 65536), vocab, rng.choice((_log(rng, 16, 8192), 64 * _log(rng, 1, 128))), dtype, rng.random() < 0.6)
        if _cost(c) <= most[op]:
            del c["name"]
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 5e13)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def _taking_part(c):
    """rows that take part: every fifth or so is left out, from the front, as a prompt is"""
    return c["rows"] - int(c["rows"] * c["skipped"])


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "score":
        n = _taking_part(c)
        return {"bytes": n * c["vocab"] * e + c["rows"] * (20 + 12 * c["top"]), "flops": 5 * n * c["vocab"]}
    if c["op"] == "score_grad":
        n = _taking_part(c)
        return {"bytes": (n + c["rows"]) * c["vocab"] * e + 28 * c["rows"], "flops": 6 * n * c["vocab"]}
    if c["op"] == "distill":
        n = _taking_part(c)
        return {"bytes": (n + c["rows"]) * c["vocab"] * e + 12 * n * c["top"] + 8 * c["rows"], "flops": 7 * n * c["vocab"]}
    if c["op"] == "norm":
        return {"bytes": c["width"] * (2 * c["rows"] + 2) * e + 8 * c["rows"], "flops": 7 * c["rows"] * c["width"]}
    if c["op"] == "norm_grad":
        return {"bytes": c["width"] * ((3 + c["add"]) * c["rows"] + 1) * e + 8 * c["rows"] + 8 * c["width"], "flops": 12 * c["rows"] * c["width"]}
    # rows of the table that some token names: token v of a log-uniform distribution has the share log(1 + 1/(v+1)) / log(V+1)
    share = torch.log1p(1 / torch.arange(1, c["vocab"] + 1, dtype=torch.float64)) / math.log(c["vocab"] + 1)
    named = float((1 - (1 - share) ** c["tokens"]).sum())
    if c["op"] == "embed":
        return {"bytes": int((named + c["tokens"]) * c["width"]) * e + 8 * c["tokens"], "flops": c["tokens"] * c["width"]}
    table = 8 * named * c["width"] if c["accumulate"] else 4 * c["vocab"] * c["width"]
    return {"bytes": int(c["tokens"] * c["width"] * e + table) + 8 * c["tokens"], "flops": 2 * c["tokens"] * c["width"]}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
IGNORE, EPS = -100, 1e-5


def prepare(case, seed):
    c = dict(case)
    dt = DTYPES[c["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def rand(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std
    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")
    s = {"case": c}
    if c["op"] in ("score", "score_grad", "distill"):
        n, V = c["rows"], c["vocab"]
        # a model's logits: most of the vocabulary far below a few likely tokens
        z = rand(n, V + c["pad"], std=2.0)
        likely = torch.randint(V, (n, 12), generator=gen, device="cuda")
        z.scatter_add_(1, likely, 6.0 + rand(n, 12, std=3.0))
        if c["masked"]:
            z[:, V - c["masked"]:V] = -math.inf
        s["buffer"] = z.to(dt)
        s["logits"] = s["buffer"][:, :V]
        skipped = n - _taking_part(c)
        if c["op"] == "distill":
            # a teacher that mostly agrees with the student, its values at the temperature of the loss
            t = 0.8 * s["logits"].float() + rand(n, V)
            if c["tail"]:
                t = torch.log_softmax(t / c["temperature"], 1)
            top = torch.topk(t, c["top"], 1)
            s["ids"], s["values"] = top.indices.contiguous(), top.values.contiguous()
            s["weight"] = torch.full((n,), 1.0 / n, device="cuda")
            s["weight"][:skipped] = 0.0
            s["row_loss"] = empty(n)
            s["d_logits"] = torch.empty_like(s["buffer"])[:, :V]
            return s
        s["tokens"] = likely[:, 0].clone()
        if c["masked"]:
            s["tokens"].clamp_(max=V - c["masked"] - 1)
        s["tokens"][:skipped] = IGNORE
        if c["op"] == "score":
            for x in ("logp", "lse", "entropy"):
                s[x] = empty(n)
            s["top_logp"], s["top_ids"] = empty(n, c["top"]), empty(n, c["top"], dtype=torch.int64)
            return s
        s["d_logp"], s["d_entropy"] = rand(n, std=1.0 / n), torch.full((n,), -0.01 / n, device="cuda")
        st = _plain_score(c, s["logits"], s["tokens"], 0)
        s["lse"], s["entropy"] = st["lse"], st["entropy"]
        s["d_logits"] = torch.empty_like(s["buffer"])[:, :V]
        return s
    if c["op"].startswith("norm"):
        n, d = c["rows"], c["width"]
        x = rand(n, d) + rand(n, 1, std=0.3)
        x[:, ::max(1, d // 5)] *= 8.0                                   # a few loud channels
        s["x"], s["gain"], s["bias"] = x.to(dt), (1 + rand(d, std=0.1)).to(dt), rand(d, std=0.1).to(dt)
        s["y"], s["mean"], s["rstd"] = empty(n, d, dtype=dt), empty(n), empty(n)
        if c["op"] == "norm_grad":
            _, s["mean"], s["rstd"] = _plain_norm(s["x"], s["gain"], s["bias"])
            s["dy"] = rand(n, d, std=1e-2).to(dt)
            s["add"] = rand(n, d, std=1e-2).to(dt) if c["add"] else None
            s["dx"], s["d_gain"], s["d_bias"] = empty(n, d, dtype=dt), empty(d), empty(d)
        return s
    n, V, d = c["tokens"], c["vocab"], c["width"]
    s["ids"] = (torch.exp(torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    # frequent words lie anywhere in a vocabulary
    s["ids"] = (s["ids"] * 7919) % V
    if c["op"] == "embed":
        s["table"], s["out"] = rand(V, d, std=0.02).to(dt), empty(n, d, dtype=dt)
    else:
        s["dy"] = rand(n, d, std=1e-3).to(dt)
        s["d_table"] = rand(V, d, std=1e-3) if c["accumulate"] else empty(V, d)
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
ORDER = ("logp", "lse", "entropy", "top_logp", "top_ids")


def _plain_score(c, logits, tokens, top):
    z = logits.float()
    part = tokens != IGNORE
    heat = c["temperature"]
    peak = z.amax(1, keepdim=True)
    d = (z - peak) / heat
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    out = {"lse": (peak / heat + log_total).squeeze(1)}
    out["entropy"] = (log_total - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True) / total).squeeze(1)
    at = torch.where(part, tokens, 0)[:, None]
    out["logp"] = (d.gather(1, at) - log_total).squeeze(1)
    out = {k: torch.where(part, v, 0.0) for k, v in out.items()}
    if top:
        column = torch.arange(z.shape[1], dtype=torch.int32, device=z.device)
        values, ids = [], []
        for _ in range(top):
            # the largest of what is left; of equal ones the first
            best = d.amax(1, keepdim=True)
            i = torch.where(d == best, column, z.shape[1]).amin(1, keepdim=True).long()
            values.append(best)
            ids.append(i)
            d.scatter_(1, i, -math.inf)
        out["top_logp"] = torch.where(part[:, None], torch.cat(values, 1) - log_total, -math.inf)
        out["top_ids"] = torch.where(part[:, None], torch.cat(ids, 1), -1)
    return {x: out[x] for x in ORDER if x in out}


def _plain_score_grad(s):
    c = s["case"]
    z, heat = s["logits"].float(), c["temperature"]
    part = (s["tokens"] != IGNORE)[:, None]
    logp = z / heat - s["lse"][:, None]
    p = torch.exp(logp)
    g, h = s["d_logp"][:, None], s["d_entropy"][:, None]
    out = p * (-g - h * (logp + s["entropy"][:, None]))
    out.scatter_add_(1, torch.where(part, s["tokens"][:, None], 0), g)
    return torch.where(part, out / heat, 0.0).to(s["logits"].dtype)


def _plain_distill(s):
    c = s["case"]
    z, heat, w = s["logits"].float(), c["temperature"], s["weight"][:, None]
    d = (z - z.amax(1, keepdim=True)) / heat
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_p = d.gather(1, s["ids"]) - torch.log(total)
    if c["tail"]:
        log_q = s["values"]
        q = torch.exp(log_q)
        rest_q = (1 - torch.exp(log_q.double()).sum(1, keepdim=True)).clamp(min=0).float()
        rest = e.scatter(1, s["ids"], 0.0)
        rest_p = rest.sum(1, keepdim=True) / total
        loss = (q * (log_q - log_p)).sum(1) + torch.where(rest_q > 0, rest_q * (torch.log(rest_q) - torch.log(rest_p)), 0.0).squeeze(1)
        mass = q.sum(1, keepdim=True) + rest_q
        grad = mass * e / total - rest_q * rest / (total * rest_p)
    else:
        t = s["values"] / heat
        t = t - t.amax(1, keepdim=True)
        log_q = t - torch.log(torch.exp(t).sum(1, keepdim=True))
        q = torch.exp(log_q)
        loss = (q * (log_q - log_p)).sum(1)
        grad = e / total
    grad.scatter_add_(1, s["ids"], -q)
    return {"row_loss": torch.where(w[:, 0] != 0, loss, 0.0), "d_logits": (grad * w / heat).to(s["logits"].dtype)}


def _plain_norm(x, gain, bias):
    f = x.float()
    mean = f.mean(1, keepdim=True)
    f = f - mean
    rstd = 1 / torch.sqrt((f * f).mean(1, keepdim=True) + EPS)
    return (f * rstd * gain.float() + bias.float()).to(x.dtype), mean.squeeze(1), rstd.squeeze(1)


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dy * s["gain"].float()
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(s["x"].dtype), "d_gain": (dy * xhat).sum(0), "d_bias": dy.sum(0)}


def _plain_embed_grad(s):
    c = s["case"]
    if not c["accumulate"]:
        s["d_table"].zero_()
    return s["d_table"].index_add_(0, s["ids"], s["dy"].float() * math.sqrt(c["width"]))


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2506_03077_b200 import binding as B
    c = s["case"]
    def workspace(nbytes):
        if "workspace" not in s:
            s["workspace"] = B.alloc_workspace(nbytes())
        return s["workspace"]
    if c["op"] == "score":
        B.token_logprobs(s["logits"], s["tokens"], workspace(B.token_logprobs_workspace_bytes), logp=s["logp"], lse=s["lse"],
                         entropy=s["entropy"], top_logp=s["top_logp"], top_ids=s["top_ids"], temperature=c["temperature"],
                         ignore_index=IGNORE)
        return {x: s[x] for x in ("logp", "lse", "entropy") + (("top_logp", "top_ids") if c["top"] else ())}
    if c["op"] == "score_grad":
        B.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], s["d_logits"], d_logp=s["d_logp"],
                                  d_entropy=s["d_entropy"], temperature=c["temperature"], ignore_index=IGNORE)
        return s["d_logits"]
    if c["op"] == "distill":
        B.distill_topk(s["logits"], s["ids"], s["values"], s["row_loss"], workspace(B.distill_topk_workspace_bytes),
                       d_logits=s["d_logits"], weight=s["weight"], temperature=c["temperature"], tail=c["tail"])
        return {"row_loss": s["row_loss"], "d_logits": s["d_logits"]}
    if c["op"] == "norm":
        B.layernorm_forward(s["x"], s["gain"], s["bias"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if c["op"] == "norm_grad":
        B.layernorm_backward(s["dy"], s["x"], s["gain"], s["mean"], s["rstd"], dx=s["dx"], d_gain=s["d_gain"], d_bias=s["d_bias"],
                             add=s["add"], workspace=workspace(lambda: B.layernorm_workspace_bytes(c["rows"], c["width"])))
        return {"dx": s["dx"], "d_gain": s["d_gain"], "d_bias": s["d_bias"]}
    if c["op"] == "embed":
        B.embedding_forward(s["table"], s["ids"], s["out"], workspace(B.embedding_workspace_bytes), scale=math.sqrt(c["width"]))
        return s["out"]
    B.embedding_backward(s["dy"], s["ids"], s["d_table"], workspace(lambda: B.embedding_backward_workspace_bytes(c["tokens"], c["vocab"], c["width"])),
                         scale=math.sqrt(c["width"]), accumulate=c["accumulate"])
    return s["d_table"]


def run(state):
    if own:
        return _own(state)
    s, c = state, state["case"]
    if c["op"] == "score":
        return _plain_score(c, s["logits"], s["tokens"], c["top"])
    if c["op"] == "score_grad":
        return _plain_score_grad(s)
    if c["op"] == "distill":
        return _plain_distill(s)
    if c["op"] == "norm":
        y, mean, rstd = _plain_norm(s["x"], s["gain"], s["bias"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["op"] == "norm_grad":
        return _plain_norm_grad(s)
    if c["op"] == "embed":
        return (s["table"][s["ids"]].float() * math.sqrt(c["width"])).to(s["table"].dtype)
    return _plain_embed_grad(s)


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_score(c, s):
    out = {x: [] for x in ORDER}
    for i in range(c["rows"]):
        if int(s["tokens"][i]) == IGNORE:
            for x in ("logp", "lse", "entropy"):
                out[x].append(torch.zeros((), dtype=torch.float64, device="cuda"))
            out["top_logp"].append(torch.full((c.get("top", 0),), -math.inf, dtype=torch.float64, device="cuda"))
            out["top_ids"].append(torch.full((c.get("top", 0),), -1, device="cuda"))
            continue
        z = s["logits"][i].double() / c["temperature"]
        lse = torch.logsumexp(z, 0)
        lp = z - lse
        out["logp"].append(lp[s["tokens"][i]])
        out["lse"].append(lse)
        out["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum())
        value, index = torch.sort(s["logits"][i].float(), descending=True, stable=True)
        out["top_ids"].append(index[:c.get("top", 0)])
        out["top_logp"].append(lp[index[:c.get("top", 0)]])
    out = {x: torch.stack(v) for x, v in out.items()}
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    f64 = torch.float64
    if c["op"] == "score":
        out = _exact_score(c, s)
        return {x: out[x] for x in (ORDER if c["top"] else ORDER[:3])}
    if c["op"] == "score_grad":
        # the formula's value for the statistics that the call is given
        out = torch.zeros(c["rows"], c["vocab"], dtype=f64, device="cuda")
        for i in range(c["rows"]):
            t = int(s["tokens"][i])
            if t == IGNORE:
                continue
            lp = s["logits"][i].double() / c["temperature"] - s["lse"][i].double()
            row = -(s["d_logp"][i].double() + s["d_entropy"][i].double() * (lp + s["entropy"][i].double())) * torch.exp2(lp / math.log(2))
            row[t] += s["d_logp"][i].double()
            out[i] = row / c["temperature"]
        return out
    if c["op"] == "distill":
        heat = c["temperature"]
        loss, grad = torch.zeros(c["rows"], dtype=f64, device="cuda"), torch.zeros(c["rows"], c["vocab"], dtype=f64, device="cuda")
        for i in range(c["rows"]):
            w = float(s["weight"][i])
            if w == 0:
                continue
            z = (s["logits"][i].double() / heat).requires_grad_()
            ids, t = s["ids"][i], s["values"][i].double()
            log_p = torch.log_softmax(z, 0)
            if c["tail"]:
                rest = torch.ones(c["vocab"], dtype=torch.bool, device="cuda")
                rest[ids] = False
                b = 1 - t.exp().sum()
                kl = torch.nn.functional.kl_div(log_p[ids], t, reduction="sum", log_target=True)
                if float(b) > 0:
                    kl = kl + b * (torch.log(b) - torch.logsumexp(log_p[rest], 0))
            else:
                kl = torch.nn.functional.kl_div(log_p[ids], torch.log_softmax(t / heat, 0), reduction="sum", log_target=True)
            g, = torch.autograd.grad(kl, z)
            loss[i], grad[i] = kl.detach(), g * (w / heat)
        return {"row_loss": loss, "d_logits": grad}
    if c["op"] == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = torch.rsqrt(var + EPS)
        return {"y": torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["gain"].double()), "mean": mean, "rstd": rstd}
    if c["op"] == "norm_grad":
        # the formula's value for the mean and the deviation that the call is given
        h = torch.addcmul(-(s["mean"].double() * s["rstd"].double())[:, None], s["x"].double(), s["rstd"].double()[:, None])
        dy = s["dy"].double()
        a = torch.einsum("nd,d->n", dy, s["gain"].double()) / c["width"]
        b = torch.einsum("nd,nd,d->n", dy, h, s["gain"].double()) / c["width"]
        dx = s["rstd"].double()[:, None] * (dy * s["gain"].double() - a[:, None] - h * b[:, None])
        return {"dx": dx if s["add"] is None else dx + s["add"].double(), "d_gain": torch.einsum("nd,nd->d", dy, h), "d_bias": dy.sum(0)}
    if c["op"] == "embed":
        return torch.nn.functional.embedding(s["ids"], s["table"]).double() * math.sqrt(c["width"])
    out = s["d_table"].double() if c["accumulate"] else torch.zeros(c["vocab"], c["width"], dtype=f64, device="cuda")
    return out.index_put_((s["ids"],), s["dy"].double() * math.sqrt(c["width"]), accumulate=True)
