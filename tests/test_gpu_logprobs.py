"""Token log-probabilities, entropy and alternatives, and their gradient, against the definitions in 64 bits.

Tolerances.  A row's S is a sum of positive terms e: each is off by the exponential's 2^-22 and by its argument's rounding,
|log2 e| 2^-24 (at most 40 of it for terms that matter), the sums by at most 170 roundings of 2^-24: log S is good to
1.5e-5.  logp and lse add roundings of their own size; the entropy adds the same share of itself.  A probability of the
gradient is exp of (z / tau - lse), off by |log p| 2^-23 + 2^-22 (at most 1.5e-5 where log p > -100; smaller p are compared
absolutely), and the result is rounded once."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16
SUM = 1.5e-5


def half_step(dt):
    return torch.finfo(dt).eps / 2


def logits_of(rows, V, dtype, pad=0, start=0, seed=0, std=3.0):
    """[rows, V] at element `start` of a buffer whose rows are V + pad apart"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = (torch.randn(rows * (V + pad) + start + 8, generator=g, device="cuda") * std).to(dtype)
    return buf[start:start + rows * (V + pad)].view(rows, V + pad)[:, :V]


def score(z, tokens, k=0, tau=1.0, ignore=-100, status=B.OK):
    n = z.shape[0]
    out = {x: torch.full((n,), 7.0, device="cuda") for x in ("logp", "lse", "entropy")}
    if tokens is None:
        out["logp"] = None
    if k:
        out["top_logp"], out["top_ids"] = torch.full((n, k), 7.0, device="cuda"), torch.full((n, k), 7, device="cuda")
    ws = B.alloc_workspace(B.token_logprobs_workspace_bytes())
    B.token_logprobs(z, tokens, ws, temperature=tau, ignore_index=ignore, **out)
    assert B.last_device_status(ws) == status
    return out


def reference(z, tokens, k, tau, ignore=-100):
    a = z.double() / tau
    lse = torch.logsumexp(a, 1)
    lp = a - lse[:, None]
    ref = {"lse": lse, "entropy": -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)}
    v, i = torch.sort(z.float(), dim=1, descending=True, stable=True)
    ref["top_ids"] = i[:, :k]
    ref["top_logp"] = lp.gather(1, i[:, :k])
    if tokens is not None:
        part = tokens != ignore
        ref["logp"] = lp.gather(1, torch.where(part, tokens, 0)[:, None]).squeeze(1)
        for x in ("logp", "lse", "entropy"):
            ref[x] = torch.where(part, ref[x], 0.0)
        ref["top_ids"] = torch.where(part[:, None], ref["top_ids"], -1)
        ref["top_logp"] = torch.where(part[:, None], ref["top_logp"], -math.inf)
    return ref


def near(got, want, share=0.0):
    """off by at most SUM, four roundings of the value, and `share` of it"""
    want = want.to(torch.float64)
    same = (got.double() == want) | (torch.isnan(got) & torch.isnan(want))
    off = (got.double() - want).abs()
    bad = ~(same | (off <= SUM + (2.0 ** -22 + share) * want.abs()))
    assert not bad.any(), (got[bad][:4], want[bad][:4])


def check(z, tokens, k, tau=1.0):
    got, ref = score(z, tokens, k, tau), reference(z, tokens, k, tau)
    near(got["lse"], ref["lse"])
    near(got["entropy"], ref["entropy"], SUM)
    if tokens is not None:
        near(got["logp"], ref["logp"])
    if k:
        assert torch.equal(got["top_ids"], ref["top_ids"])
        near(got["top_logp"], ref["top_logp"])
    return got


def tokens_of(n, V, seed=1, ignored=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(V, (n,), generator=g, device="cuda")
    t[:ignored] = -100
    return t


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,V,k,pad,start,tau", [
    (1, 1, 1, 0, 0, 1.0), (2, 2, 2, 0, 1, 1.0), (5, 7, 7, 1, 3, 0.5), (3, 128, 128, 0, 0, 1.0), (4, 200, 128, 5, 2, 0.7),
    (1, 4097, 20, 0, 1, 1.0), (9, 2049, 1, 3, 0, 2.0), (33, 32003, 16, 0, 0, 1.0), (600, 5003, 5, 1, 7, 1.0),
    (1, 152064, 128, 0, 0, 1.0), (3, 152064, 20, 64, 0, 0.7), (40, 152061, 64, 0, 5, 1.0), (2, 600001, 100, 0, 0, 1.0), (300, 32000, 0, 0, 0, 1.0)])
def test_rows(rows, V, k, pad, start, tau, dtype):
    check(logits_of(rows, V, dtype, pad, start), tokens_of(rows, V, ignored=rows // 4), k, tau)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["constant", "zeros", "ascending", "descending", "few", "comb", "stripe", "ends"])
@pytest.mark.parametrize("rows,V", [(2, 33000), (300, 20011), (1, 300)])
def test_lists_of_hard_rows(kind, rows, V, dtype):
    """ties, orders and crowds: the lists have to be those of a stable sort"""
    i = torch.arange(V, device="cuda")
    z = {"constant": torch.full((V,), 1.5, device="cuda"), "zeros": torch.where(i % 3 == 0, -0.0, 0.0), "ascending": i / V * 9,
         "descending": -i / V * 9, "few": (i % 5).float(), "comb": ((i // 4) % 256 == 17) * (5 + i / V), "stripe": ((i // 4) % 256 < 4) * (i % 977) / 100,
         "ends": ((i < 3) | (i >= V - 3)) * 4.0}[kind].to(dtype)
    z = z.expand(rows, V).contiguous()
    for k in (1, 20, 128):
        check(z, None, k)


def test_masked_and_broken_rows():
    inf, V = math.inf, 5000
    z = logits_of(7, V, F32)
    z[0] = -inf
    z[1, 17:] = -inf
    z[2, :] = -inf
    z[2, 4321] = 2.0
    z[3, 100] = math.nan
    z[4, 200] = inf
    z[5, 1000:] = torch.finfo(F32).min
    tokens = torch.tensor([3, 2, 4321, 1, 200, 9, 10], device="cuda")
    got = score(z, tokens, 20)
    assert got["lse"][0] == -inf and got["logp"][0] == -inf and got["entropy"][0] == 0 and (got["top_logp"][0] == -inf).all()
    assert torch.equal(got["top_ids"][0], torch.arange(20, device="cuda"))
    for r in (3, 4):
        assert all(torch.isnan(got[x][r]) for x in ("lse", "logp", "entropy")) and torch.isnan(got["top_logp"][r]).all()
        assert (got["top_ids"][r] == -1).all()
    ref = reference(z[[1, 2, 5, 6]], tokens[[1, 2, 5, 6]], 20, 1.0)
    for x in ("lse", "logp", "entropy", "top_logp"):
        near(got[x][[1, 2, 5, 6]], ref[x], SUM)
    assert torch.equal(got["top_ids"][[1, 2, 5, 6]], ref["top_ids"])
    assert got["entropy"][2] == 0 and got["logp"][2] == 0
    d = torch.empty_like(z)
    one = torch.ones(7, device="cuda")
    B.token_logprobs_backward(z, tokens, got["lse"], got["entropy"], d, d_lse=one, d_entropy=one)
    assert (d[0] == 0).all() and torch.isnan(d[3, 100]) and torch.isfinite(d[[1, 2, 5, 6]]).all() and (d[1, 17:] == 0).all()


def test_tokens_outside_the_vocabulary():
    z = logits_of(5, 1000, BF)
    tokens = torch.tensor([3, -100, 1000, 5, -1], device="cuda")
    got = score(z, tokens, 4, status=B.E_BAD_LABEL)
    ref = reference(z, torch.tensor([3, -100, -100, 5, -100], device="cuda"), 4, 1.0)
    near(got["logp"], ref["logp"])
    assert torch.equal(got["top_ids"], ref["top_ids"])


def test_large_logits_keep_their_digits():
    """an offset that both sides see changes lse alone"""
    z = logits_of(4, 3001, F32, std=1.0).mul(64).round().div(64)        # multiples of 1/64: sums with 4096 are exact
    t = tokens_of(4, 3001)
    a, b = score(z, t, 8), score(z + 4096, t, 8)
    for x in ("logp", "entropy", "top_logp", "top_ids"):
        assert torch.equal(a[x], b[x])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,V,pad,start,tau,inplace", [
    (1, 1, 0, 0, 1.0, False), (3, 7, 1, 1, 0.5, True), (5, 4099, 3, 2, 1.0, False), (17, 32003, 0, 0, 0.7, True), (2, 152064, 0, 0, 2.0, False)])
def test_gradient(rows, V, pad, start, tau, inplace, dtype):
    z, t = logits_of(rows, V, dtype, pad, start), tokens_of(rows, V, ignored=rows // 4)
    fw = score(z, t, 0, tau)
    g = torch.Generator(device="cuda").manual_seed(5)
    gp, gl, gh = (torch.randn(rows, generator=g, device="cuda") for _ in range(3))
    part = (t != -100)[:, None]
    zd = z.double().clone().requires_grad_()
    lp = torch.log_softmax(zd / tau, 1)
    at = torch.where(part, t[:, None], 0)
    total = (part[:, 0] * (gp * lp.gather(1, at)[:, 0] + gl * torch.logsumexp(zd / tau, 1) - gh * (lp.exp() * lp).sum(1))).sum()
    want, = torch.autograd.grad(total, zd)
    p, ref = lp.detach().exp(), lp.detach()
    size = p * (gp.abs() + gl.abs() + gh.abs() * (fw["entropy"] + 1))[:, None] + p * ref.abs() * gh.abs()[:, None]
    size = (size + torch.zeros_like(size).scatter(1, at, gp.abs()[:, None].double())) / tau
    d = z if inplace else torch.full_like(z, 7.0)
    other = None
    if pad:                                  # a gradient whose rows start elsewhere
        other = torch.full((rows, V), 7.0, device="cuda", dtype=dtype)
        B.token_logprobs_backward(z, t, fw["lse"], fw["entropy"], other, d_logp=gp, d_lse=gl, d_entropy=gh, temperature=tau)
    B.token_logprobs_backward(z, t, fw["lse"], fw["entropy"], d, d_logp=gp, d_lse=gl, d_entropy=gh, temperature=tau)
    # (the lse and entropy that it is given are off by SUM and their rounding)
    bound = (half_step(dtype) + 3 * SUM + 2.0 ** -22 * (1 + fw["lse"].abs()[:, None])) * size + 1e-30
    assert ((d.double() - want).abs() <= bound).all()
    assert other is None or torch.equal(other, d)


def test_single_gradients_and_differences():
    z = logits_of(3, 50, F32, std=1.0)
    t = tokens_of(3, 50)
    fw = score(z, t)
    one = torch.ones(3, device="cuda")
    for name in ("logp", "lse", "entropy"):
        d = torch.empty_like(z)
        B.token_logprobs_backward(z, t if name == "logp" else None, fw["lse"], fw["entropy"], d, **{"d_" + name: one})
        h = 2.0 ** -6
        for j in (0, 17, 49):
            up, down = z.clone(), z.clone()
            up[:, j] += h
            down[:, j] -= h
            slope = (reference(up, t, 1, 1.0)[name] - reference(down, t, 1, 1.0)[name]) / (2 * h)
            assert ((d[:, j].double() - slope).abs() <= 1e-4).all()          # h^2 of third derivatives below 1 / 6 each


def test_rows_behind_and_between_are_left(dtype=BF):
    buf = torch.full((10, 1000), 3.0, device="cuda", dtype=dtype)
    z = logits_of(6, 900, dtype)
    t = tokens_of(6, 900)
    fw = score(z, t)
    B.token_logprobs_backward(z, t, fw["lse"], None, buf[2:8, 11:911], d_logp=torch.ones(6, device="cuda"))
    assert (buf[:2] == 3).all() and (buf[8:] == 3).all() and (buf[:, :11] == 3).all() and (buf[:, 911:] == 3).all()


def test_many_rows_with_tokens_outside():
    """more than one block looks through"""
    z = logits_of(20000, 40, BF)
    t = tokens_of(20000, 40, ignored=3)
    check(z, t, 3)
    t[19999] = 40
    got = score(z, t, 3, status=B.E_BAD_LABEL)
    assert got["logp"][19999] == 0 and (got["top_ids"][19999] == -1).all()
    t[19999] = 5
    score(z, t, 3)
