"""Attention with a sliding window and sink keys, forward and backward, against numpy in 64 bits.

Bounds, per element.  bf16: the products S and dP are formed from exact bf16 operands and summed in fp32; P and dS are
rounded once as operands (2^-8 each, relative), outputs once (2^-8); exp2, lse and the fp32 sums stay below 2^-14 of the
terms' magnitudes (|S| <= 40 in base 2: 40 * 2^-23 from the scaled score and the lse, 2^-22 from ex2.approx, sums of up to
1000 terms).  delta is formed from the forward's rounded O, so its error is |dO| times that of O.  fp32 runs: the same
with 2^-14 replaced by 2^-17 (scores below 30: __expf is off by 2^-21 + 2^-24 |x| relative) and no operand rounding."""
import numpy as np
import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu

FENCE = 5.0
BF, F32 = torch.bfloat16, torch.float32


def visible(n, q0, window, sinks):
    t, j = np.arange(q0, q0 + n)[:, None], np.arange(q0 + n)[None]
    return (j <= t) & ((t - j < window) | (j < sinks))


class Case:
    def __init__(self, n, q0, Hq, Hkv, dh, window, sinks, dtype=BF, seed=0, std=1.0):
        self.n, self.q0, self.Hq, self.Hkv, self.dh, self.window, self.sinks, self.dtype = n, q0, Hq, Hkv, dh, window, sinks, dtype
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda rows, heads: (torch.randn(rows, heads, dh, generator=g, device="cuda") * std).to(dtype)
        self.q, self.k, self.v, self.do = rand(n, Hq), rand(q0 + n, Hkv), rand(q0 + n, Hkv), rand(n, Hq)

    def fenced(self, *shape, dtype, fill=float("nan")):
        count = int(np.prod(shape))
        buf = torch.full((count + 256,), FENCE, dtype=dtype, device="cuda")
        buf[:count] = fill
        return buf[:count].view(*shape), buf

    def forward(self, engine=0):
        o, ob = self.fenced(*self.q.shape, dtype=self.dtype)
        lse, lb = self.fenced(self.Hq, self.n, dtype=F32)
        B.attention_window_forward(self.q, self.k, self.v, self.q0, self.window, self.sinks, o, lse, engine=engine)
        assert bool((ob[o.numel():] == FENCE).all()) and bool((lb[lse.numel():] == FENCE).all())
        return o, lse

    def backward(self, o, lse, grad_dtype=F32, accumulate=False, fill=float("nan"), engine=0):
        outs, bufs = [], []
        for t in (self.q, self.k, self.v):
            x, b = self.fenced(*t.shape, dtype=grad_dtype, fill=fill)
            outs.append(x)
            bufs.append(b)
        need = B.attention_window_workspace_bytes(self.n, self.q0, self.Hq, self.Hkv, self.dh, self.window, self.sinks)
        ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
        B.attention_window_backward(self.q, self.k, self.v, o, self.do, lse, self.q0, self.window, self.sinks, *outs, ws[:need],
                                    accumulate=accumulate, engine=engine)
        for x, b in zip(outs, bufs):
            assert bool((b[x.numel():] == FENCE).all())
        assert bool((ws[need:] == 7).all())
        assert B.last_device_status(ws) == B.OK
        return outs

    def reference(self):
        """o, lse, dq, dk, dv and the bounds of each."""
        f = lambda t: t.double().cpu().numpy()
        q, k, v, do = f(self.q), f(self.k), f(self.v), f(self.do)
        see, G, scale = visible(self.n, self.q0, self.window, self.sinks), self.Hq // self.Hkv, self.dh ** -0.5
        half = 2.0 ** -8 if self.dtype == BF else 0.0
        tiny = 2.0 ** -14 if self.dtype == BF else 2.0 ** -17
        out = {x: np.zeros_like(y) for x, y in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
        out["lse"] = np.zeros((self.Hq, self.n))
        e = {x: np.zeros_like(y) for x, y in out.items()}
        for h in range(self.Hq):
            g = h // G
            s = q[:, h] @ k[:, g].T * scale
            s[~see] = -np.inf
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            l = p.sum(1, keepdims=True)
            p /= l
            out["lse"][h], e["lse"][h] = (top + np.log(l))[:, 0], 2.0 ** -18 * (1 + np.abs(top[:, 0]) + np.log(see.sum(1)))
            o = p @ v[:, g]
            out["o"][:, h], e["o"][:, h] = o, (half + tiny) * (p @ np.abs(v[:, g])) + tiny * np.abs(o)
            eo = e["o"][:, h] + half * (np.abs(o) + e["o"][:, h])          # of the rounded output
            d = do[:, h]
            dp, delta = d @ v[:, g].T, (d * o).sum(1, keepdims=True)
            ed = (np.abs(d) * eo).sum(1, keepdims=True) + tiny * (np.abs(d) * np.abs(o)).sum(1, keepdims=True)
            ds = p * (dp - delta) * scale
            es = half * np.abs(ds) + p * scale * (ed + tiny * (np.abs(d) @ np.abs(v[:, g]).T + np.abs(delta)))
            es = es * (1 + half)
            out["dq"][:, h], e["dq"][:, h] = ds @ k[:, g], es @ np.abs(k[:, g]) + tiny * (np.abs(ds) @ np.abs(k[:, g]))
            out["dk"][:, g] += ds.T @ q[:, h]
            e["dk"][:, g] += es.T @ np.abs(q[:, h]) + tiny * (np.abs(ds).T @ np.abs(q[:, h]))
            out["dv"][:, g] += p.T @ d
            e["dv"][:, g] += (half + tiny) * (p.T @ np.abs(d))
        return out, e

    def check(self, name, got, ref, err, extra=0.0):
        g = got.double().cpu().numpy()
        h = 2.0 ** -8 if got.dtype == BF else 2.0 ** -23
        bound = err + h * (np.abs(ref) + err) + 1e-30 + extra
        bad = ~(np.abs(g - ref) <= bound)
        assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {ref[bad][0]} +- {bound[bad][0]}"


def run(case, engines=(0,), grads=(F32,)):
    ref, err = case.reference()
    for engine in engines:
        o, lse = case.forward(engine)
        case.check("o", o, ref["o"], err["o"])
        case.check("lse", lse, ref["lse"], err["lse"])
        for gd in grads:
            for name, x in zip(("dq", "dk", "dv"), case.backward(o, lse, gd, engine=engine)):
                case.check(f"{name} engine {engine} {gd}", x, ref[name], err[name])
        # adding: to what the accumulators hold (dq is overwritten)
        dq, dk, dv = case.backward(o, lse, F32, accumulate=True, fill=0.25, engine=engine)
        case.check("dq", dq, ref["dq"], err["dq"])
        case.check("dk +=", dk, ref["dk"] + 0.25, err["dk"], 2.0 ** -24)
        case.check("dv +=", dv, ref["dv"] + 0.25, err["dv"], 2.0 ** -24)


SHAPES = [
    # n, q0, window, sinks
    (1, 0, 1, 0), (1, 500, 100, 3), (2, 0, 2, 1), (5, 300, 64, 0), (127, 0, 20, 0), (128, 0, 128, 4), (129, 0, 129, 0),
    (130, 126, 1, 0), (200, 56, 127, 130), (256, 128, 128, 1), (300, 0, 1000, 4), (333, 700, 200, 0), (333, 700, 200, 5),
    (511, 513, 300, 129), (600, 0, 40, 128), (600, 0, 40, 113), (600, 0, 40, 16), (600, 300, 70, 290), (700, 0, 33, 17), (700, 100, 255, 256), (640, 0, 640, 640), (640, 0, 5, 10000),
]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,q0,window,sinks", SHAPES)
def test_tensor_core_shapes(n, q0, window, sinks, dh):
    run(Case(n, q0, 4, 2, dh, window, sinks), engines=(0,), grads=(F32, BF))


# (rows, heads): more (128-row tile, head) items than the GPU holds at half load, so that the forward walks them with persistent
# CTAs; tiles of 1, 2, 4, 16 and 32 heads of a group
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(32, 32), (28, 4), (24, 12), (32, 8), (32, 2), (64, 1)])
def test_many_items(Hq, Hkv, dh):
    for n, q0, window, sinks in ((777, 100, 90, 3), (801, 0, 300, 70)):
        run(Case(n, q0, Hq, Hkv, dh, window, sinks), grads=(BF,))


# few rows: all heads of a group in one tile (47 does not divide into 128 rows), key tiles dealt to a cluster, some of whose
# CTAs see nothing of a row
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (16, 1), (47, 1), (150, 1), (6, 2), (8, 8)])
def test_few_rows(Hq, Hkv, dh):
    for n, q0, window, sinks in ((1, 0, 1, 0), (1, 999, 1000, 0), (1, 777, 100, 400), (3, 1500, 640, 1), (9, 1000, 3, 700), (20, 1, 20, 0)):
        run(Case(n, q0, Hq, Hkv, dh, window, sinks), grads=(BF, F32))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (6, 6), (14, 2), (3, 3)])
def test_head_layouts(Hq, Hkv):
    run(Case(300, 150, Hq, Hkv, 64, 100, 2), engines=(0, 2), grads=(BF,))
    run(Case(270, 0, Hq, Hkv, 128, 130, 0), engines=(0, 2), grads=(BF,))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,q0,window,sinks", SHAPES[::2])
def test_cuda_cores(n, q0, window, sinks, dh):
    run(Case(n, q0, 4, 2, dh, window, sinks, F32))
    run(Case(n, q0, 2, 1, dh, window, sinks, BF), engines=(1,), grads=(BF,))


def test_sink_sums_joined_from_segments():
    """Long enough that the query tiles of the sink tiles are cut, on both engines."""
    run(Case(1500, 0, 2, 1, 64, 100, 3), engines=(0, 1), grads=(F32, BF))
    run(Case(1300, 200, 2, 2, 128, 64, 140), engines=(0,), grads=(BF,))
    run(Case(900, 0, 2, 1, 64, 40, 70, F32))


def test_a_window_over_everything_is_causal_attention():
    c = Case(700, 300, 4, 2, 128, 5000, 3)
    o, lse = c.forward()
    want, want_lse = torch.empty_like(o), torch.empty_like(lse)
    B.attention_forward(c.q, c.k, c.v, c.q0, want, want_lse)
    # The two kernels take their maxima over 64 and over 128 keys at a time, so their P are rounded against different
    # references: each is within its own bound of the exact result (P to 2^-8 of sum p |v|), not of the other's bits.
    ref, err = c.reference()
    for x, y in ((o, lse), (want, want_lse)):
        c.check("o", x, ref["o"], err["o"])
        c.check("lse", y, ref["lse"], err["lse"])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_chunks_add_up_to_the_whole(dtype):
    """Rows in chunks, last to first, as the streamed backward walks them: dk and dv accumulate over the chunks."""
    n, W, S = 900, 200, 5
    whole = Case(n, 0, 4, 2, 64, W, S, dtype)
    ref, err = whole.reference()
    dk, dv = torch.zeros_like(whole.k, dtype=F32), torch.zeros_like(whole.v, dtype=F32)
    for begin in range(n // 256 * 256, -1, -256):
        end = min(n, begin + 256)
        c = Case(end - begin, begin, 4, 2, 64, W, S, dtype)
        c.q, c.k, c.v, c.do = whole.q[begin:end].contiguous(), whole.k[:end].contiguous(), whole.v[:end].contiguous(), whole.do[begin:end].contiguous()
        o, lse = c.forward()
        whole.check("o", o, ref["o"][begin:end], err["o"][begin:end])
        ws = B.alloc_workspace(B.attention_window_workspace_bytes(c.n, c.q0, 4, 2, 64, W, S))
        dq = torch.empty_like(c.q, dtype=F32)
        B.attention_window_backward(c.q, c.k, c.v, o, c.do, lse, begin, W, S, dq, dk[:end], dv[:end], ws, accumulate=True)
        whole.check("dq", dq, ref["dq"][begin:end], err["dq"][begin:end])
    whole.check("dk", dk, ref["dk"], err["dk"], 2.0 ** -20)
    whole.check("dv", dv, ref["dv"], err["dv"], 2.0 ** -20)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_keys_that_no_query_sees_are_not_read(dtype):
    """NaN in every row of k and v that lies in no key tile of the chunk's span."""
    c = Case(100, 1000, 2, 1, 64, 50, 2, dtype)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    tile = 128 if dtype == BF else 32
    lo = (1000 - 50 + 1) // tile * tile
    c.k[tile:lo] = float("nan")
    c.v[tile:lo] = float("nan")
    o2, lse2 = c.forward()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(grads, c.backward(o2, lse2)):
        assert torch.equal(a, b)
    assert bool((grads[1][2:1000 - 49] == 0).all()) and bool((grads[2][2:1000 - 49] == 0).all())


@pytest.mark.parametrize("dtype,dh,Hq,Hkv,n,q0,window,sinks", [
    (BF, 64, 8, 2, 300, 1000, 333, 5), (BF, 128, 8, 2, 300, 1000, 333, 5), (BF, 128, 28, 4, 5, 1000, 333, 70),
    (BF, 64, 16, 1, 1, 500, 100, 129), (BF, 128, 2, 2, 130, 250, 200, 0), (BF, 128, 32, 32, 700, 430, 300, 33),
    (BF, 64, 32, 32, 700, 430, 300, 33), (BF, 128, 1, 1, 200, 100, 60, 30), (BF, 64, 8, 2, 200, 100, 60, 30),
    (BF, 64, 40, 1, 700, 200, 170, 20), (F32, 64, 4, 2, 100, 300, 77, 5), (F32, 128, 2, 1, 40, 100, 90, 7)])
def test_rows_that_no_query_sees_may_hold_anything(dtype, dh, Hq, Hkv, n, q0, window, sinks):
    """NaN, infinities and the largest values in every row of k and v that no query of the chunk sees, also where such a row
    shares a tile with visible ones."""
    c = Case(n, q0, Hq, Hkv, dh, window, sinks, dtype)
    see = torch.from_numpy(visible(n, q0, window, sinks).any(0)).cuda()
    c.k[~see], c.v[~see] = 0.0, 0.0
    o, lse = c.forward()
    want = [o, lse] + list(c.backward(o, lse)) + ([] if dtype == F32 else list(c.backward(o, lse, BF)))
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).max):
        c.k[~see], c.v[~see] = bad, -bad
        o, lse = c.forward()
        got = [o, lse] + list(c.backward(o, lse)) + ([] if dtype == F32 else list(c.backward(o, lse, BF)))
        for a, b in zip(want, got):
            assert torch.equal(a, b)
    assert bool((got[3][~see] == 0).all()) and bool((got[4][~see] == 0).all())


def test_large_scores():
    """Scores of several hundred: the running maximum grows by large steps, weights of far keys vanish."""
    c = Case(300, 100, 2, 1, 128, 150, 4, std=3.0)
    ref, err = c.reference()
    o, lse = c.forward()
    # |S| up to 300 in base 2: the bound of the exponent's argument grows with it
    c.check("o", o, ref["o"], err["o"] * 4)
    c.check("lse", lse, ref["lse"], err["lse"])
    for name, x in zip(("dq", "dk", "dv"), c.backward(o, lse)):
        c.check(name, x, ref[name], err[name] * 4)


def test_results_are_reproducible():
    c = Case(1500, 0, 4, 2, 64, 100, 3)
    o, lse = c.forward()
    first = c.backward(o, lse, BF)
    for _ in range(3):
        o2, lse2 = c.forward()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert all(torch.equal(a, b) for a, b in zip(first, c.backward(o, lse, BF)))


def test_capture_and_other_stream():
    c = Case(400, 100, 4, 2, 128, 150, 4)
    o, lse = c.forward()
    want = c.backward(o, lse, BF)
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    got = [torch.zeros_like(x) for x in want]
    ws = B.alloc_workspace(B.attention_window_workspace_bytes(400, 100, 4, 2, 128, 150, 4))
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        B.attention_window_forward(c.q, c.k, c.v, 100, 150, 4, o2, lse2)
        B.attention_window_backward(c.q, c.k, c.v, o2, c.do, lse2, 100, 150, 4, *got, ws)
    for _ in range(2):
        for x in [o2, lse2] + got:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip(want, got))
    o2.zero_()
    torch.cuda.synchronize()
    B.attention_window_forward(c.q, c.k, c.v, 100, 150, 4, o2, lse2, stream=s)
    s.synchronize()
    assert torch.equal(o, o2)


def test_calls_at_once_and_replayed():
    """Calls of every way to cut the work (clusters, segments, persistent CTAs), each with its own workspace: on streams of
    their own at the same time, and captured into graphs that are replayed at the same time, give the bits that they give
    alone."""
    cases = [Case(5, 2000, 28, 4, 128, 1024, 4), Case(20, 3000, 16, 1, 64, 2500, 0), Case(2000, 0, 16, 1, 128, 2000, 0),
             Case(700, 300, 32, 8, 64, 200, 33), Case(1, 900, 8, 8, 128, 900, 0), Case(200, 100, 40, 1, 64, 60, 30)]
    want = []
    for c in cases:
        o, lse = c.forward()
        want.append([o, lse] + list(c.backward(o, lse, BF)))
    out = [[torch.empty_like(x) for x in w] for w in want]
    ws = [B.alloc_workspace(B.attention_window_workspace_bytes(c.n, c.q0, c.Hq, c.Hkv, c.dh, c.window, c.sinks)) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]

    def call(c, x, w):
        B.attention_window_forward(c.q, c.k, c.v, c.q0, c.window, c.sinks, x[0], x[1])
        B.attention_window_backward(c.q, c.k, c.v, x[0], c.do, x[1], c.q0, c.window, c.sinks, x[2], x[3], x[4], w)

    def same():
        torch.cuda.synchronize()
        for a, b, w in zip(want, out, ws):
            assert all(torch.equal(x, y) for x, y in zip(a, b)) and B.last_device_status(w) == B.OK
            for y in b:
                y.fill_(float("nan"))
        torch.cuda.synchronize()

    torch.cuda.synchronize()
    for _ in range(3):
        for c, x, w, s in zip(cases, out, ws, streams):
            with torch.cuda.stream(s):
                call(c, x, w)
    same()
    graphs = []
    for c, x, w in zip(cases, out, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(c, x, w)
        graphs.append(g)
    same_before = [x[0].isnan().all() for x in out]
    assert all(bool(b) for b in same_before)              # captured, not run
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    same()


def test_gradient_against_differences():
    """Directional derivatives of sum(O * dO) by central differences of the fp32 forward."""
    c = Case(70, 30, 2, 1, 64, 25, 3, F32)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    loss = lambda: (c.forward()[0].double() * c.do.double()).sum().item()
    g = torch.Generator(device="cuda").manual_seed(3)
    for t, d in zip((c.q, c.k, c.v), grads):
        base, way = t.clone(), torch.randn(t.shape, generator=g, device="cuda")
        h = 2.0 ** -8
        values = []
        for s in (1, -1):
            t.copy_(base + s * h * way)
            values.append(loss())
        t.copy_(base)
        slope = (d.double() * way.double()).sum().item()
        size = (d.double().abs() * way.double().abs()).sum().item()
        # fp32 outputs of about 9000 terms near 1 over 2h, and the third derivative's h^2
        assert abs((values[0] - values[1]) / (2 * h) - slope) <= size * 2e-3 + 1e-2


def test_refusals():
    c = Case(64, 32, 4, 2, 64, 16, 1)
    o, lse = torch.empty_like(c.q), torch.empty(4, 64, device="cuda")
    for kw in (dict(k=c.k[1:]), dict(v=c.v.float()), dict(o=o[:10]), dict(lse=lse[:, :3].contiguous()), dict(q=c.q.transpose(0, 1)),
               dict(q0=31), dict(k=c.k.cpu()), dict(o=o.float())):
        a = dict(q=c.q, k=c.k, v=c.v, q0=32, window=16, sinks=1, o=o, lse=lse)
        a.update(kw)
        with pytest.raises(ValueError):
            B.attention_window_forward(**a)
    for kw in (dict(window=0), dict(sinks=-1), dict(engine=7)):
        a = dict(q=c.q, k=c.k, v=c.v, q0=32, window=16, sinks=1, o=o, lse=lse)
        a.update(kw)
        with pytest.raises(B.StreamBPError):
            B.attention_window_forward(**a)
    ws = B.alloc_workspace(B.attention_window_workspace_bytes(64, 32, 4, 2, 64, 16, 1))
    g = [torch.empty_like(x) for x in (c.q, c.k, c.v)]
    with pytest.raises(B.StreamBPError):
        B.attention_window_backward(c.q, c.k, c.v, o, c.do, lse, 32, 16, 1, *g, ws, accumulate=True)      # bf16 accumulators
    with pytest.raises(B.StreamBPError):
        B.attention_window_backward(c.q, c.k, c.v, o, c.do, lse, 32, 16, 1, *g, ws[:256])
    with pytest.raises(ValueError):
        B.attention_window_backward(c.q, c.k, c.v, o, c.do, lse, 32, 16, 1, g[0], g[1].float(), g[2], ws)
