"""Distillation over the range of temperatures and of gaps between listed and unlisted tokens, against the definition in 64 bits.

The definition here has the unlisted tokens' p_j / p_r as a softmax of their own, so that it holds at any gap.  Tolerances are
those of test_gpu_distill.py: log p good to 1.5e-5 and its rounding, the terms Q p, q and q_r p / p_r each to 3e-5 of
themselves, one rounding of the result; probabilities below 2^-126 count as 0 (1e-30 beside them)."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from helpers import TOL
from test_gpu_distill import distill
from test_gpu_logprobs import BF, F32, SUM, half_step
from test_gpu_model_ends import Head, relative

pytestmark = pytest.mark.gpu
GAPS = [0.0, 14.0, 60.0, 80.0, 86.0, 87.0, 87.5, 88.0, 90.0, 95.0, 126.0, 200.0, 1000.0, 20000.0]
f32 = lambda x: float(torch.tensor(x, dtype=F32))


def definition(z, ids, values, w, tau, tail):
    """losses, gradients and the sizes of the gradients' terms"""
    losses, grads, sizes = [], [], []
    for r in range(z.shape[0]):
        a = z[r].double() / tau
        lp = torch.log_softmax(a, 0)
        c, t = ids[r], values[r].double()
        q = t.exp() if tail else torch.softmax(t / tau, 0)
        q_of = torch.zeros_like(a).index_add_(0, c, q)
        loss = (torch.special.xlogy(q, q) - torch.where(q > 0, q * lp[c], 0.0)).sum()
        rest = a > -math.inf
        rest[c] = False
        rest_q = max(0.0, 1 - float(q.sum())) if tail and rest.any() else 0.0
        Q = float(q.sum()) + rest_q
        of_rest = torch.zeros_like(a)
        if rest_q > 0:
            loss = loss + rest_q * (math.log(rest_q) - (torch.logsumexp(a[rest], 0) - torch.logsumexp(a, 0)))
            of_rest[rest] = rest_q * torch.softmax(a[rest], 0)
        losses.append(loss)
        grads.append((Q * lp.exp() - q_of - of_rest) * (w / tau))
        sizes.append((Q * lp.exp() + q_of + of_rest) * (w / tau))
    return torch.stack(losses), torch.stack(grads), torch.stack(sizes)


def compare(z, ids, values, tau, tail, w=1.0):
    want_l, want_g, size = definition(z, ids, values, w, tau, tail)
    loss, d = distill(z, ids, values, torch.full((z.shape[0],), w, device="cuda"), tau, tail)
    Q = values.double().exp().sum(1) + 1 if tail else 1.0
    assert ((loss.double() - want_l).abs() <= (2 * SUM + 2.0 ** -22 * 40) * Q + 2.0 ** -23 * want_l.abs()).all()
    assert ((d.double() - want_g).abs() <= (half_step(d.dtype) + 2 * SUM) * size + 1e-30 * (1 + w / tau)).all()
    own = z.clone()
    assert torch.equal(distill(own, ids, values, torch.full((z.shape[0],), w, device="cuda"), tau, tail, own)[1], d)
    return loss, d


def rows_with_gaps(V, tau, dtype, masked, k=6, seed=0):
    """one row a gap: its first listed tokens, three of them neighbours, lie that many tau above the others' scale"""
    n = len(GAPS)
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(n, V, generator=g, device="cuda") * tau
    ids = torch.randint(V - 3, (n, k), generator=g, device="cuda")
    ids[:, 1], ids[:, 2] = ids[:, 0] + 1, ids[:, 0] + 2
    if masked:
        z[:, ::2] = -math.inf
    up = torch.randn(n, k, generator=g, device="cuda") * tau + torch.tensor(GAPS, device="cuda")[:, None] * tau
    z.scatter_(1, ids, up)
    return z.to(dtype), ids


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tau", [1.0, f32(0.05), 2.0 ** -20, 2.0 ** 20, f32(7.3)])
@pytest.mark.parametrize("V", [60, 5003, 40001])
def test_a_remainder_far_below_the_listed_tokens(V, tau, dtype, masked):
    z, ids = rows_with_gaps(V, tau, dtype, masked)
    for rest in (0.4, 0.05, 1e-3):
        q = torch.tensor([0.3, 0.25, 0.2, 0.1, 0.1, 0.05], dtype=torch.float64) * (1 - rest)
        values = q.log().float().cuda().expand(z.shape[0], 6).contiguous()
        loss, d = compare(z, ids, values, tau, True)
        # a divergence, and not below 0, where no token is listed twice: (a + b) log(a + b) > a log a + b log b
        once = ids.sort(1).values.diff(dim=1).ne(0).all(1)
        assert (loss[once] >= -1e-4).all() and torch.isfinite(d).all() and (V < 100 or once.sum() > 10)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tau", [1.0, f32(0.05)])
def test_unlisted_tokens_of_their_own_range(tau, dtype):
    """far below the listed ones, and far apart from one another; one alone; none; in rows of many blocks"""
    V = 70001
    z = torch.full((5, V), -math.inf, device="cuda")
    z[0] = torch.linspace(-120, 0, V, device="cuda") * tau
    z[1] = torch.linspace(-500, -100, V, device="cuda") * tau
    z[2, 69999] = -300 * tau
    z[4] = torch.where(torch.arange(V, device="cuda") % 1000 == 7, -150 * tau, -400 * tau)
    ids = torch.tensor([5, 30000, 30001, 70000], device="cuda").repeat(5, 1)
    z.scatter_(1, ids, torch.tensor([1.0, 3.0, 0.0, 2.0], device="cuda").mul(tau).repeat(5, 1))
    z = z.to(dtype)
    values = torch.tensor([0.2, 0.3, 0.1, 0.1], dtype=torch.float64).log().float().cuda().repeat(5, 1)
    compare(z, ids, values, tau, True, 0.125)


@pytest.mark.parametrize("tail", [False, True])
def test_unlisted_tokens_above_the_listed(tail):
    """the student is sure of something that the teacher does not list"""
    for tau in (1.0, f32(0.05)):
        z, ids = rows_with_gaps(5003, tau, F32, False)
        q = torch.tensor([0.3, 0.2, 0.2, 0.1, 0.1, 0.05], dtype=torch.float64)
        values = q.log().float().cuda().expand(z.shape[0], 6).contiguous()
        compare(-z, ids, values if tail else values * tau, tau, tail)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("chunk,group", [(64, 1), (48, 3)])
def test_the_streamed_head_with_a_remainder_far_below(chunk, group, dtype):
    h = Head(dtype)
    h.H[:, 0] = 4
    h.W[:, 0] = 0
    h.W[:4, 0] = 60                                # these four some two hundred above all others
    ids = torch.arange(4, device="cuda").repeat(h.T, 1)
    q = torch.tensor([0.4, 0.2, 0.1, 0.1], dtype=torch.float64, device="cuda")
    values = q.log().float().repeat(h.T, 1)
    w = torch.full((h.T,), 1.0 / h.T, device="cuda")
    loss, row, dH, dW, dg = h.distill(ids, values, w, chunk, group, tail=True)
    H, g, W = (x.double().requires_grad_() for x in (h.H, h.g, h.W))
    z = h.logits(H, g, W)
    assert (z[:, :4].amin(1) - z[:, 4:].amax(1) > 100).all()
    lp, rest = torch.log_softmax(z, 1), 1 - float(q.sum())
    want = (q * (q.log() - lp[:, :4])).sum(1) + rest * (math.log(rest) - (torch.logsumexp(z[:, 4:], 1) - torch.logsumexp(z, 1)))
    total = (want * w.double()).sum()
    assert abs(loss.item() - total.item()) <= (1e-4 if dtype == F32 else 2e-2) * abs(total.item())
    for got, ref in zip((dH, dg, dW), torch.autograd.grad(total, (H, g, W))):
        assert relative(got, ref) <= TOL[dtype]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("chunk,group", [(64, 1), (32, 2)])
def test_chunks_without_entries_are_not_read(chunk, group, dtype):
    """rows without entries take no part, whatever their hidden states are, as those of weight 0"""
    h = Head(dtype)
    h.H[64:128] = math.inf
    ids = torch.randint(h.V, (h.T, 5), device="cuda")
    values = torch.zeros(h.T, 5, device="cuda")
    one, some = torch.full((h.T,), 1.0 / h.T, device="cuda"), torch.full((h.T,), 1.0 / h.T, device="cuda")
    some[64:128] = 0
    want = h.distill(ids, values, some, chunk, group)
    ids[64:128] = -1
    got = h.distill(ids, values, one, chunk, group)
    for a, b in zip(got, want):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    h.H.fill_(math.nan)
    ids.fill_(-1)
    for x in h.distill(ids, values, one, chunk, group):       # (weights are there: this is no call without any)
        assert (x == 0).all()
    h.distill(ids, values, 0 * one, chunk, group, status=B.E_NO_VALID_LABELS)
    ids[70, 2] = h.V
    h.distill(ids, values, one, chunk, group, status=B.E_BAD_LABEL)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,V", [(5, 4099), (3, 100001), (700, 3000)])
def test_rows_without_entries(n, V, tail):
    """in blocks alone and in clusters, all ids absent or outside, beside rows with a single one at any place of the list"""
    g = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn(n, V, generator=g, device="cuda")
    z[1::2] = math.nan
    for k in (1, 33, 128):
        ids = torch.full((n, k), -1, device="cuda")
        ids[0::2, k - 1] = torch.randint(V, (len(ids[0::2]),), generator=g, device="cuda")
        values = torch.full((n, k), -0.5, device="cuda")
        w = torch.ones(n, device="cuda")
        loss, d = distill(z, ids, values, w, 1.0, tail)
        assert (loss[1::2] == 0).all() and (d[1::2] == 0).all()
        want_l, want_g, size = definition(z[0:3:2], ids[0:3:2, k - 1:], values[0:3:2, k - 1:], 1.0, 1.0, tail)
        assert ((loss[0:3:2].double() - want_l).abs() <= 4 * SUM + 2.0 ** -22 * 40 + 2.0 ** -23 * want_l.abs()).all()
        assert ((d[0:3:2].double() - want_g).abs() <= (half_step(F32) + 2 * SUM) * size + 1e-30).all()
        ids[1, 0] = V
        again = distill(z, ids, values, w, 1.0, tail, status=B.E_BAD_LABEL)
        assert torch.equal(again[0], loss) and torch.equal(again[1], d)


@pytest.mark.parametrize("gap", [0.0, 88.0, 300.0])
def test_gradients_far_below_by_differences(gap):
    z = torch.randn(2, 40, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    ids = torch.tensor([[3, 17, 4], [39, 0, 20]], device="cuda")
    z.scatter_add_(1, ids, torch.full((2, 3), gap, device="cuda"))
    values = torch.tensor([0.5, 0.2, 0.1], dtype=torch.float64).log().float().cuda().repeat(2, 1)
    _, d = distill(z, ids, values, None, 1.0, True)
    h = 2.0 ** -8
    for j in (0, 3, 20, 25):
        up, down = z.double(), z.double()
        up[:, j] += h
        down[:, j] -= h
        slope = (definition(up, ids, values, 1.0, 1.0, True)[0] - definition(down, ids, values, 1.0, 1.0, True)[0]) / (2 * h)
        # h^2 / 6 of third derivatives of log-sums (below 1 / 2 each, times Q + q_r), the terms' 3e-5, losses of up to 100 in 64 bits
        assert ((d[:, j].double() - slope).abs() <= 2e-6 * 1.2 + 3e-5 * 2 + 1e-10).all()
