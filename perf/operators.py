"""What is measured of the operators around the streamed backward: attention with a sliding window and a few first
tokens that stay visible (forward and backward), the matrix product with bias, activation and residual in its
epilogue (and the gradient of that epilogue), and the clipped AdamW step over many tensors.

Each operator has a plain form made of elementary torch operations (`own` false) and the call a user makes of the
library (`own` true).  Cases are dicts of plain values; `listed()` names the fixed ones, `draw()` spreads over the
same ranges."""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _attn(name, op, n, q0, heads, kv_heads, dim, window, sinks, dtype="bf16"):
    return {"name": name, "op": op, "n": n, "q0": q0, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "window": window, "sinks": sinks, "dtype": dtype}


def _linear(name, op, m, n, k, act, bias=True, residual=False, pre=True, dtype="bf16"):
    return {"name": name, "op": op, "m": m, "n": n, "k": k, "act": act, "bias": bias, "residual": residual,
            "pre": pre, "dtype": dtype}


def _adamw(name, elements, tensors, state, param="bf16", master=False, clip=True):
    return {"name": name, "op": "adamw", "elements": elements, "tensors": tensors, "state": state, "param": param,
            "master": master, "clip": clip}


def listed():
    return [
        # one chunk of a streamed layer deep in a 16k sequence: 32 / 8 heads of 128, a window of 4096 keys
        _attn("attn_fwd_chunk", "attn_fwd", 2048, 14336, 32, 8, 128, 4096, 4),
        # a whole sequence under a short window, heads of 64: little arithmetic per byte
        _attn("attn_fwd_short_window", "attn_fwd", 16384, 0, 32, 8, 64, 128, 1),
        # the ragged last chunk of a sequence: a few rows against the window, latency counts
        _attn("attn_fwd_few_rows", "attn_fwd", 5, 4091, 28, 4, 128, 1024, 4),
        # one chunk of a streamed backward, seven query heads to a key head
        _attn("attn_bwd_chunk", "attn_bwd", 1024, 7168, 28, 4, 128, 2048, 16),
        # a whole sequence of odd length: every query adds to the gradient of the sink keys
        _attn("attn_bwd_whole", "attn_bwd", 8191, 0, 32, 8, 64, 512, 4),
        # up projection of one chunk: bias and GELU, pre-activation kept for the backward
        _linear("linear_up", "linear", 2048, 14336, 4096, "gelu_tanh"),
        # output projection of a ragged chunk: bias and residual, nothing kept
        _linear("linear_out_ragged", "linear", 777, 3584, 3584, "none", residual=True, pre=False),
        # the gradient of the epilogue of the up projection
        _linear("linear_grad_up", "linear_grad", 2048, 14336, 4096, "gelu_tanh"),
        # the same for a short chunk of odd width
        _linear("linear_grad_ragged", "linear_grad", 333, 2731, 1024, "silu"),
        # one layer of 233 M parameters, moments in 8 bits, gradients clipped by their global norm
        _adamw("adamw_layer_8bit", 233_000_000, 12, "mx8"),
        # a model of many small tensors, moments in 32 bits, fp32 master weights
        _adamw("adamw_many_32bit", 40_000_000, 150, "f32", master=True),
        # gains and biases only: the smallest step
        _adamw("adamw_small_32bit", 60_000, 20, "f32", param="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 8, 128), (28, 4, 128), (4, 2, 64), (32, 8, 64), (8, 8, 128), (16, 1, 64), (12, 4, 128))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("attn_fwd", "attn_bwd", "linear", "linear_grad", "adamw")}
    while True:
        op = rng.choice(("attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd", "linear", "linear_grad", "adamw"))
        if op.startswith("attn"):
            f32 = rng.random() < 0.2
            h, g, d = (4, 2, 64) if f32 else rng.choice(HEADS)
            n = _log(rng, 1 if op == "attn_fwd" else 2, 512 if f32 else 16384)
            q0 = rng.choice((0, _log(rng, 1, 16384))) if not f32 else rng.randrange(0, 256)
            c = _attn("", op, n, q0, h, g, d, _log(rng, 8, 512 if f32 else 4096), rng.choice((0, 1, 4, 16, 100, 200)),
                      "f32" if f32 else "bf16")
        elif op == "linear":
            f32 = rng.random() < 0.15
            act = rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu"))
            size = (lambda: 8 * _log(rng, 4, 128)) if f32 else (lambda: 8 * _log(rng, 16, 1800))
            c = _linear("", op, _log(rng, 1, 512 if f32 else 8192), size() - rng.choice((0, 0, 3)), size(), act,
                        rng.random() < 0.8, rng.random() < 0.5, act != "none" and rng.random() < 0.7, "f32" if f32 else "bf16")
        elif op == "linear_grad":
            c = _linear("", op, _log(rng, 1, 8192), _log(rng, 64, 20000), 1024, rng.choice(("relu", "gelu", "gelu_tanh", "silu")),
                        dtype=rng.choice(("bf16", "bf16", "f32")))
        else:
            param = rng.choice(("bf16", "bf16", "f32"))
            c = _adamw("", _log(rng, 2000, 200_000_000), _log(rng, 1, 200), rng.choice(("mx8", "f32")), param,
                       param == "bf16" and rng.random() < 0.5, rng.random() < 0.7)
        if _cost(c) <= most[op]:
            del c["name"]
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 1.5e15)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def _pairs(c):
    """(visible (query, key) pairs of one head, keys that some query sees)"""
    n, q0, w, s = c["n"], c["q0"], c["window"], c["sinks"]
    i = torch.arange(q0, q0 + n, dtype=torch.int64)
    pairs = int((torch.clamp(i + 1, max=w) + torch.clamp(i + 1 - w, min=0, max=s)).sum())
    first = max(0, q0 - w + 1)
    return pairs, q0 + n - first + min(s, first)


def work(case):
    c = case
    if c["op"].startswith("attn"):
        pairs, keys = _pairs(c)
        e = 2 if c["dtype"] == "bf16" else 4
        qo, kv, lse = c["n"] * c["heads"] * c["dim"] * e, keys * c["kv_heads"] * c["dim"] * e, 4 * c["n"] * c["heads"]
        if c["op"] == "attn_fwd":
            return {"bytes": 2 * qo + 2 * kv + lse, "flops": 4 * c["dim"] * pairs * c["heads"]}
        return {"bytes": 4 * qo + 2 * kv + lse + 2 * (c["q0"] + c["n"]) * c["kv_heads"] * c["dim"] * e,
                "flops": 10 * c["dim"] * pairs * c["heads"]}
    if c["op"] == "linear":
        e = 2 if c["dtype"] == "bf16" else 4
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": e * (m * k + n * k + m * n * (1 + c["residual"] + c["pre"]) + n * c["bias"]), "flops": 2 * m * n * k}
    if c["op"] == "linear_grad":
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 3 * e * c["m"] * c["n"] + 4 * c["n"], "flops": 20 * c["m"] * c["n"]}
    p = 2 if c["param"] == "bf16" else 4
    # the step itself; with moments in 8 bits also the reading of the updated moments as values
    state = 16 if c["state"] == "f32" else 2 * (2 + 2 / 32) + 2 * (1 + 1 / 32 + 2)
    return {"bytes": c["elements"] * (4 + (p if c["master"] else 2 * p) + (8 if c["master"] else 0) + state), "flops": 20 * c["elements"]}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8}
STEP, MAX_NORM, DECAY = 7, 1.0, 0.1


def _sizes(c):
    """Sizes of the tensors of an AdamW case: a few that hold most of it, the others small, most of them odd."""
    n = max(1, min(c["tensors"], c["elements"] // 8))
    share = [1.0 / (1 + (i * 5) % 7) ** 2 for i in range(n)]
    return [max(1, int(c["elements"] * s / sum(share)) - (i % 3)) for i, s in enumerate(share)]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def rand(*shape, dtype, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)
    if c["op"].startswith("attn"):
        dt, n, kv = DTYPES[c["dtype"]], c["n"], c["q0"] + c["n"]
        s = {"case": c, "q": rand(n, c["heads"], c["dim"], dtype=dt), "k": rand(kv, c["kv_heads"], c["dim"], dtype=dt),
             "v": rand(kv, c["kv_heads"], c["dim"], dtype=dt)}
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(c["heads"], n, device="cuda")
        if c["op"] == "attn_bwd":
            s["d_o"] = rand(n, c["heads"], c["dim"], dtype=dt)
            s["o"], s["lse"] = _plain_attention(c, s["q"], s["k"], s["v"])
            s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
        return s
    if c["op"] == "linear":
        dt, m, n, k = DTYPES[c["dtype"]], c["m"], c["n"], c["k"]
        return {"case": c, "a": rand(m, k, dtype=dt), "w": rand(n, k, dtype=dt, std=k ** -0.5),
                "bias": rand(n, dtype=dt, std=0.5) if c["bias"] else None, "residual": rand(m, n, dtype=dt) if c["residual"] else None,
                "y": torch.empty(m, n, dtype=dt, device="cuda"), "z": torch.empty(m, n, dtype=dt, device="cuda") if c["pre"] else None}
    if c["op"] == "linear_grad":
        dt, m, n = DTYPES[c["dtype"]], c["m"], c["n"]
        return {"case": c, "dy": rand(m, n, dtype=dt), "z": rand(m, n, dtype=dt), "dz": torch.empty(m, n, dtype=dt, device="cuda"),
                "dbias": torch.empty(n, device="cuda")}
    # AdamW: parameters, gradients and moments of all tensors lie in flat buffers, each tensor on a boundary of 64
    # elements (the layout of the per-layer gradient bucket); what is between them stays zero
    sizes, offsets, total = _sizes(c), [], 0
    for z in sizes:
        offsets.append(total)
        total += -(-z // 64) * 64
    inside = torch.zeros(total // 64, 64, dtype=torch.bool, device="cuda")
    for z, o in zip(sizes, offsets):
        inside.view(-1)[o:o + z] = True
    inside = inside.view(-1)
    decay = torch.zeros(total // 64, device="cuda")
    for i, (z, o) in enumerate(zip(sizes, offsets)):
        decay[o // 64:(o + z + 63) // 64] = 0.0 if i % 3 == 2 else DECAY     # gains and biases do not decay
    s = {"case": c, "sizes": sizes, "offsets": offsets, "decay": decay}
    s["grad"] = rand(total, dtype=torch.float32, std=3e-4) * inside
    master = rand(total, dtype=torch.float32, std=0.02) * inside
    s["param"] = master.to(DTYPES[c["param"]])
    s["master"] = master if c["master"] else None
    del master
    m = rand(total, dtype=torch.float32, std=1e-4) * inside
    u = (rand(total, dtype=torch.float32, std=3e-4).abs() + 1e-6) * inside     # root of the second moment
    if c["state"] == "f32":
        s["m"], s["v"] = m, u * u
    else:
        s["m"], s["m_scale"] = _mx8(m)
        s["v"], s["v_scale"] = _mx8(u, keep=True)
        s["m_out"], s["v_out"] = (torch.empty(total, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s["norm"], s["scale"] = torch.ones(1, device="cuda"), torch.ones(1, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _band(c, q, k, v):
    """Scores of every query against the keys of its block's band and the sink keys, softmax over the visible ones.

    Queries go in blocks of B rows; a block sees the window + B - 1 keys that end with its last row.  Columns are
    those keys and then the sinks.  Returns the probabilities, the row sums' logarithm and what made them."""
    n, q0, H, G = c["n"], c["q0"], c["kv_heads"], c["heads"] // c["kv_heads"]
    kv = q0 + n
    W, S = min(c["window"], kv), min(c["sinks"], kv)
    B = max(1, min(n, 512, max(64, 1 << (W - 1).bit_length())))
    nb, L = -(-n // B), W + B - 1
    dev = q.device
    start = q0 + torch.arange(nb, device=dev) * B - (W - 1)
    key = torch.cat([start[:, None] + torch.arange(L, device=dev), torch.arange(S, device=dev).expand(nb, S)], 1)   # [nb, L + S]
    row = (torch.arange(nb, device=dev) * B)[:, None] + torch.arange(B, device=dev)
    pos = (q0 + row)[:, :, None]
    near = (key[:, None] >= 0) & (key[:, None] <= pos) & (pos - key[:, None] < c["window"])
    far = (key[:, None] <= pos) & (pos - key[:, None] >= c["window"])
    is_sink = torch.arange(L + S, device=dev) >= L
    visible = torch.where(is_sink, far, near) & (row < n)[:, :, None]                 # [nb, B, L + S]
    at = key.clamp(0, kv - 1).reshape(-1)
    kb = k.float()[at].view(nb, L + S, H, -1).permute(0, 2, 1, 3)                     # [nb, H, L + S, d]
    vb = v.float()[at].view(nb, L + S, H, -1).permute(0, 2, 1, 3)
    qb = _blocks(c, q, nb, B)
    s = (qb @ kb.transpose(2, 3)).view(nb, H, G, B, L + S) * c["dim"] ** -0.5
    s = torch.where(visible[:, None, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    s = torch.exp(s - top)
    total = s.sum(-1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1).permute(1, 2, 0, 3).reshape(H * G, nb * B)[:, :n]
    return s.div_(total).view(nb, H, G * B, L + S), lse, qb, kb, vb, at


def _blocks(c, x, nb, B):
    """[n, heads, d] as [blocks, kv heads, heads of the group x B rows, d] in 32 bits, zero rows behind the last"""
    H, G, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    f = torch.zeros(nb * B, H * G, d, device=x.device)
    f[:c["n"]] = x
    return f.view(nb, B, H, G, d).permute(0, 2, 3, 1, 4).reshape(nb, H, G * B, d)


def _rows(c, x, nb, B):
    """the way back"""
    H, G, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    return x.view(nb, H, G, B, d).permute(0, 3, 1, 2, 4).reshape(nb * B, H * G, d)[:c["n"]]


def _plain_attention(c, q, k, v):
    p, lse, _, _, vb, _ = _band(c, q, k, v)
    nb = p.shape[0]
    B = p.shape[2] // (c["heads"] // c["kv_heads"])
    return _rows(c, p @ vb, nb, B).to(q.dtype).contiguous(), lse.contiguous()


def _plain_attention_grad(c, q, k, v, d_o):
    p, _, qb, kb, vb, at = _band(c, q, k, v)
    nb = p.shape[0]
    B = p.shape[2] // (c["heads"] // c["kv_heads"])
    db = _blocks(c, d_o, nb, B)
    dv = p.transpose(2, 3) @ db                                                       # [nb, H, L + S, d]
    ds = db @ vb.transpose(2, 3)
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * c["dim"] ** -0.5
    dk = ds.transpose(2, 3) @ qb
    dq = _rows(c, ds @ kb, nb, B)
    shape = (k.shape[0], c["kv_heads"], c["dim"])
    back = lambda x: torch.zeros(shape, device=k.device).index_add_(0, at, x.permute(0, 2, 1, 3).reshape(-1, *shape[1:]))  # noqa: E731
    return dq.to(q.dtype), back(dk).to(k.dtype), back(dv).to(v.dtype)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _mx8(x, keep=False):
    """Blocks of 32 values as e4m3 codes and one power of two: 2^(floor(log2 of the largest magnitude) - 7), as the
    byte of a biased exponent.  `keep`: a value that is not zero does not become zero."""
    b = x.view(-1, 32)
    e = (b.abs().amax(1).view(torch.int32) >> 23).sub(7).clamp(min=1)
    y = b * ((254 - e) << 23).view(torch.float32)[:, None]
    if keep:
        y = torch.where((b > 0) & (y < 2.0 ** -9), 2.0 ** -9, y)
    return y.to(torch.float8_e4m3fn).view(torch.uint8).view(-1), e.to(torch.uint8)


def _mx8_values(codes, scale):
    v = codes.view(torch.float8_e4m3fn).float().view(-1, 32) * (scale.int() << 23).view(torch.float32)[:, None]
    return v.view(-1)


def _plain_adamw(s):
    c, h = s["case"], HYPER
    g = s["grad"]
    if c["clip"]:
        s["norm"] = g.double().square().sum().sqrt().float().view(1)
        s["scale"] = (MAX_NORM / (s["norm"] + 1e-6)).clamp(max=1.0)
        g = g * s["scale"]
    mx8 = c["state"] == "mx8"
    m = _mx8_values(s["m"], s["m_scale"]) if mx8 else s["m"]
    v = _mx8_values(s["v"], s["v_scale"]).square_() if mx8 else s["v"]
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    u = v.sqrt()
    p = (s["master"] if c["master"] else s["param"]).float().view(-1, 64)
    p = p * (1 - h["lr"] * s["decay"])[:, None]
    move = m / (u / math.sqrt(1 - h["beta2"] ** STEP) + h["eps"])
    p = p.view(-1) - h["lr"] / (1 - h["beta1"] ** STEP) * move
    s["param"].copy_(p)
    if c["master"]:
        s["master"].copy_(p)
    if mx8:
        s["m"], s["m_scale"] = _mx8(m)
        s["v"], s["v_scale"] = _mx8(u, keep=True)
        m, v = (_mx8_values(s[x], s[x + "_scale"]).to(torch.bfloat16) for x in ("m", "v"))
    else:
        s["m"], s["v"] = m, v
    out = {"param": s["param"], "m": m, "v": v}
    return out | ({"master": s["master"]} if c["master"] else {}) | ({"norm": s["norm"], "scale": s["scale"]} if c["clip"] else {})


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2506_03077_b200 import binding as B
    c = s["case"]
    if c["op"] == "attn_fwd":
        B.attention_window_forward(s["q"], s["k"], s["v"], c["q0"], c["window"], c["sinks"], s["o"], s["lse"])
        return {"o": s["o"], "lse": s["lse"]}
    if c["op"] == "attn_bwd":
        if "workspace" not in s:
            s["workspace"] = B.alloc_workspace(B.attention_window_workspace_bytes(
                c["n"], c["q0"], c["heads"], c["kv_heads"], c["dim"], c["window"], c["sinks"]))
        B.attention_window_backward(s["q"], s["k"], s["v"], s["o"], s["d_o"], s["lse"], c["q0"], c["window"], c["sinks"],
                                    s["dq"], s["dk"], s["dv"], s["workspace"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if c["op"] == "linear":
        B.gemm_epilogue(s["a"], s["w"], s["y"], bias=s["bias"], activation=c["act"], residual=s["residual"], pre=s["z"])
        return {"y": s["y"]} | ({"z": s["z"]} if c["pre"] else {})
    if c["op"] == "linear_grad":
        if "workspace" not in s:
            s["workspace"] = B.alloc_workspace(B.gemm_epilogue_workspace_bytes(c["m"], c["n"]))
        B.gemm_epilogue_backward(s["dy"], s["z"], c["act"], s["dz"], s["dbias"], s["workspace"])
        return {"dz": s["dz"], "dbias": s["dbias"]}
    mx8 = c["state"] == "mx8"
    if "plan" not in s:
        tensors = []
        for z, o in zip(s["sizes"], s["offsets"]):
            t = {x: s[x][o:o + z] for x in ("param", "grad", "m", "v")}
            if c["master"]:
                t["master"] = s["master"][o:o + z]
            if mx8:
                t |= {x: s[x][o // 32:(o + z + 31) // 32] for x in ("m_scale", "v_scale")}
            tensors.append(t | {"weight_decay": 0.0 if len(tensors) % 3 == 2 else DECAY})
        s["plan"] = B.AdamWPlan(tensors)
        s["workspace"] = B.alloc_workspace(B.grad_norm_workspace_bytes())
    if c["clip"]:
        B.grad_norm(s["plan"], MAX_NORM, s["norm"], s["scale"], s["workspace"])
    B.adamw_step(s["plan"], HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], STEP, grad_scale=s["scale"] if c["clip"] else None)
    out = {"param": s["param"]} | ({"master": s["master"]} if c["master"] else {}) | ({"norm": s["norm"], "scale": s["scale"]} if c["clip"] else {})
    if mx8:
        B.mx8_decode(s["m"], s["m_scale"], s["m_out"])
        B.mx8_decode(s["v"], s["v_scale"], s["v_out"])
        return out | {"m": s["m_out"], "v": s["v_out"]}
    return out | {"m": s["m"], "v": s["v"]}


def run(state):
    if own:
        return _own(state)
    s, c = state, state["case"]
    if c["op"] == "attn_fwd":
        o, lse = _plain_attention(c, s["q"], s["k"], s["v"])
        return {"o": o, "lse": lse}
    if c["op"] == "attn_bwd":
        dq, dk, dv = _plain_attention_grad(c, s["q"], s["k"], s["v"], s["d_o"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if c["op"] == "linear":
        z = s["a"].float() @ s["w"].float().T
        if c["bias"]:
            z = z + s["bias"].float()
        y = _act(z, c["act"])
        if c["residual"]:
            y = y + s["residual"].float()
        dt = s["y"].dtype
        return {"y": y.to(dt)} | ({"z": z.to(dt)} if c["pre"] else {})
    if c["op"] == "linear_grad":
        dz = s["dy"].float() * _act_slope(s["z"].float(), c["act"])
        return {"dz": dz.to(s["dz"].dtype), "dbias": dz.sum(0)}
    return _plain_adamw(s)


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"].startswith("attn"):
        n, q0, kv, G = c["n"], c["q0"], c["q0"] + c["n"], c["heads"] // c["kv_heads"]
        t, j = torch.arange(q0, kv, device="cuda")[:, None], torch.arange(kv, device="cuda")[None]
        hidden = ~((j <= t) & ((t - j < c["window"]) | (j < c["sinks"])))
        o, lse = torch.zeros(n, c["heads"], c["dim"], dtype=torch.float64, device="cuda"), torch.zeros(c["heads"], n, dtype=torch.float64, device="cuda")
        dq, dk, dv = (torch.zeros_like(s[x], dtype=torch.float64) for x in ("q", "k", "v"))
        for h in range(c["heads"]):
            q, k, v = s["q"][:, h].double(), s["k"][:, h // G].double(), s["v"][:, h // G].double()
            a = (q @ k.T / math.sqrt(c["dim"])).masked_fill_(hidden, -math.inf)
            lse[h] = torch.logsumexp(a, 1)
            a = torch.exp_(a - lse[h][:, None])
            o[:, h] = a @ v
            if c["op"] == "attn_bwd":
                g = s["d_o"][:, h].double()
                dv[:, h // G] += a.T @ g
                g = a * (g @ v.T - (g * o[:, h]).sum(1, keepdim=True)) / math.sqrt(c["dim"])
                dq[:, h] = g @ k
                dk[:, h // G] += g.T @ q
        return {"o": o, "lse": lse} if c["op"] == "attn_fwd" else {"dq": dq, "dk": dk, "dv": dv}
    if c["op"] == "linear":
        z = torch.einsum("mk,nk->mn", s["a"].double(), s["w"].double())
        z = z if s["bias"] is None else z + s["bias"].double()
        f = torch.nn.functional
        y = {"none": lambda: z, "relu": lambda: f.relu(z), "gelu": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"),
             "silu": lambda: f.silu(z)}[c["act"]]()
        y = y if s["residual"] is None else y + s["residual"].double()
        return {"y": y} | ({"z": z} if c["pre"] else {})
    if c["op"] == "linear_grad":
        f = torch.nn.functional
        z = s["z"].double().requires_grad_()
        y = {"relu": lambda: f.relu(z), "gelu": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"), "silu": lambda: f.silu(z)}[c["act"]]()
        dz, = torch.autograd.grad(y, z, s["dy"].double())
        return {"dz": dz, "dbias": dz.sum(0)}
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    g, out = s["grad"].double(), {}
    if c["clip"]:
        norm = torch.linalg.vector_norm(g)
        scale = torch.minimum(torch.ones_like(norm), MAX_NORM / (norm + 1e-6))
        out = {"norm": norm.view(1), "scale": scale.view(1)}
        g = g * scale
    def values(x):
        e = torch.pow(2.0, s[x + "_scale"].double() - 127).repeat_interleave(32)
        return s[x].view(torch.float8_e4m3fn).double() * e
    m, v = (values("m"), values("v") ** 2) if c["state"] == "mx8" else (s["m"].double(), s["v"].double())
    m, v = torch.lerp(g, m, b1), torch.lerp(g ** 2, v, b2)
    p = (s["param"] if s["master"] is None else s["master"]).double()
    p = p - HYPER["lr"] * s["decay"].double().repeat_interleave(64) * p
    p -= HYPER["lr"] * (m / (1 - b1 ** STEP)) / ((v / (1 - b2 ** STEP)).sqrt() + HYPER["eps"])
    out |= {"param": p} | ({"master": p} if c["master"] else {})
    def held(x, positive):
        """the nearest values that 4 significant bits and the block's power of two can hold"""
        b = x.view(-1, 32)
        one = torch.exp2(torch.floor(torch.log2(b.abs().amax(1, keepdim=True).clamp(min=2.0 ** -119))) - 7).clamp(min=2.0 ** -126)
        r = b / one
        unit = torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3)
        r = torch.round(r / unit) * unit
        if positive:
            r = torch.where((b > 0) & (r < 2.0 ** -9), 2.0 ** -9, r)
        return (r * one).view(-1)
    return out | ({"m": m, "v": v} if c["state"] == "f32" else {"m": held(m, False), "v": held(v.sqrt(), True)})
