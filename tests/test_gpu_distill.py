"""Distillation from a teacher's top logits against the definition in 64 bits (autograd).

Tolerances.  log p is good to 1.5e-5 (the sums' bound of the scoring tests) and its rounding; the loss weighs it with the q.
The gradient's terms Q p, q and q_r p / p_r are each good to 3e-5 of themselves, and the result is rounded once."""
import math

import pytest
import torch

from paper_2506_03077_b200 import binding as B
from test_gpu_logprobs import BF, F32, SUM, half_step, logits_of

pytestmark = pytest.mark.gpu


def teacher(z, k, tau, tail, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = 0.8 * z.float() + torch.randn(z.shape, generator=g, device="cuda")
    if tail:
        t = torch.log_softmax(t / tau, 1)
    top = torch.topk(t, k, 1)
    return top.indices.contiguous(), top.values.contiguous()


def distill(z, ids, values, w=None, tau=1.0, tail=False, d="new", status=B.OK):
    loss = torch.full((z.shape[0],), 7.0, device="cuda")
    d = torch.full_like(z, 7.0) if isinstance(d, str) else d
    ws = B.alloc_workspace(B.distill_topk_workspace_bytes())
    B.distill_topk(z, ids, values, loss, ws, d_logits=d, weight=w, temperature=tau, tail=tail)
    assert B.last_device_status(ws) == status
    return loss, d


def reference(z, ids, values, w, tau, tail):
    """losses, gradients and the sizes of the gradients' terms, in 64 bits"""
    n, V = z.shape
    losses, grads, sizes = [], [], []
    for r in range(n):
        a = (z[r].double() / tau).requires_grad_()
        lp = torch.log_softmax(a, 0)
        on = (ids[r] >= 0) & (ids[r] < V)
        c, t = ids[r][on], values[r][on].double()
        weight = 1.0 if w is None else float(w[r])
        if weight == 0 or c.numel() == 0:
            losses.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            grads.append(torch.zeros(V, dtype=torch.float64, device="cuda"))
            sizes.append(grads[-1])
            continue
        q = t.exp() if tail else torch.softmax(t / tau, 0)
        loss = (torch.special.xlogy(q, q) - q * lp[c]).sum()
        rest = torch.ones(V, dtype=torch.bool, device="cuda")
        rest[c] = False
        rest &= a.detach() > -math.inf
        rest_q = max(0.0, 1 - float(q.sum())) if tail and rest.any() else 0.0
        size = lp.detach().exp() * (float(q.sum()) + rest_q)
        if rest_q > 0:
            log_rest = torch.logsumexp(lp[rest], 0)
            loss = loss + rest_q * (math.log(rest_q) - log_rest)
            size = size + rest * lp.detach().exp() * (rest_q / log_rest.detach().exp())
        size = size.index_add(0, c, q)
        g, = torch.autograd.grad(loss, a)
        losses.append(loss.detach())
        grads.append(torch.nan_to_num(g) * (weight / tau))
        sizes.append(size * abs(weight) / tau)
    return torch.stack(losses), torch.stack(grads), torch.stack(sizes)


def check(z, ids, values, w=None, tau=1.0, tail=False, d="new"):
    keep = z.clone()
    want_l, want_g, size = reference(keep, ids, values, w, tau, tail)
    loss, d = distill(z, ids, values, w, tau, tail, d)
    Q = values.double().exp().sum(1) + 1 if tail else 1.0
    assert ((loss.double() - want_l).abs() <= (2 * SUM + 2.0 ** -22 * 40) * Q + 2.0 ** -23 * want_l.abs()).all()
    assert ((d.double() - want_g).abs() <= (half_step(d.dtype) + 2 * SUM) * size + 1e-30).all()
    return loss, d


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,V,k,pad,start,tau", [
    (1, 1, 1, 0, 0, 1.0), (2, 2, 1, 0, 1, 1.0), (3, 129, 128, 1, 3, 0.5), (5, 4099, 8, 5, 1, 2.0), (7, 5003, 100, 0, 0, 1.0),
    (2, 152064, 32, 0, 0, 2.0), (40, 152061, 20, 3, 0, 1.0), (320, 10007, 16, 0, 0, 1.0), (3, 393216, 64, 0, 0, 1.0), (3, 300000, 5, 1, 1, 1.0)])
def test_rows(rows, V, k, pad, start, tau, dtype, tail):
    z = logits_of(rows, V, dtype, pad, start)
    ids, values = teacher(z, k, tau, tail)
    w = torch.rand(rows, device="cuda") + 0.1
    w[rows // 2:rows // 2 + rows // 4] = 0
    _, d = check(z, ids, values, w, tau, tail)
    # into the logits themselves, and into rows that start elsewhere
    other = torch.full((rows, V), 7.0, device="cuda", dtype=dtype)
    distill(z, ids, values, w, tau, tail, other)
    _, same = distill(z, ids, values, w, tau, tail, z)
    assert torch.equal(other, d) and torch.equal(same, d)


@pytest.mark.parametrize("tail", [False, True])
def test_lists_with_gaps_and_repeats(tail):
    z = logits_of(6, 3001, F32)
    ids, values = teacher(z, 12, 1.0, tail)
    ids[0, 3:] = -1
    ids[1] = -1                                    # no entries: the row takes no part
    ids[2, 5] = ids[2, 0]                          # one token three times
    ids[2, 9] = ids[2, 0]
    ids[3, 0] = 0
    ids[3, 1] = 3000
    values[4, 6:] = -math.inf                      # listed, but with q = 0
    if tail:
        values[2] -= 2.0
    loss, d = check(z, ids, values, None, 1.0, tail)
    assert loss[1] == 0 and (d[1] == 0).all()


def test_ids_outside_the_vocabulary():
    z = logits_of(4, 1000, BF)
    ids, values = teacher(z, 5, 1.0, False)
    bad = ids.clone()
    bad[1, 2], bad[2, 0], bad[3, 4] = 1000, -2, -1
    w = torch.tensor([1.0, 0.0, 0.5, 0.5], device="cuda")
    got = distill(z, bad, values, w, status=B.E_BAD_LABEL)
    bad[2, 0] = -1
    bad[1] = ids[1]
    want = distill(z, bad, values, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    bad[1, 2] = 1000                               # in a row that takes no part: nobody minds
    distill(z, bad, values, w)


def test_masked_and_broken_rows():
    z = logits_of(7, 2000, F32)
    z[0, 100:] = -math.inf
    z[1, 5] = math.nan
    z[2, 6] = math.inf
    z[4] = -math.inf
    ids = torch.arange(8, device="cuda").repeat(7, 1) + 2
    ids[3] += 500
    z[3, 505] = -math.inf                          # listed with q > 0: the loss is infinite, the gradient is not
    values = torch.log_softmax(torch.randn(7, 20, device="cuda"), 1)[:, :8].contiguous()
    z[6, 10:] = -math.inf                          # nothing left for the tail but two tokens ...
    z[6, :2] = -math.inf                           # ... and not these
    for tail in (False, True):
        w = torch.tensor([1.0, 1, 1, 1, 1, 0, 1], device="cuda")
        z[5] = math.nan                            # of weight 0
        loss, d = distill(z, ids, values, w, tail=tail)
        assert torch.isnan(loss[1:3]).all() and torch.isnan(d[1:3]).all() and torch.isinf(loss[3]) and torch.isinf(loss[4])
        assert torch.isfinite(d[[0, 3, 4, 5, 6]]).all() and (d[5] == 0).all() and loss[5] == 0
        assert (d[0, 100:] == 0).all()
        want_l, want_g, size = reference(z[[0, 6]], ids[[0, 6]], values[[0, 6]], None, 1.0, tail)
        assert ((loss[[0, 6]].double() - want_l).abs() <= 3e-4).all()
        assert ((d[[0, 6]].double() - want_g).abs() <= 1e-4 * size + 1e-30).all()


def test_a_tail_of_almost_nothing():
    """the rest's mass is a difference on the teacher's side, a sum on the student's"""
    z = logits_of(3, 5000, F32, std=0.1)
    ids = torch.arange(4, device="cuda").repeat(3, 1)
    z[:, :4] += 14.0
    q = torch.tensor([[0.25, 0.25, 0.25, 0.2499], [0.4, 0.3, 0.2, 0.0999], [0.7, 0.1, 0.1, 0.1]], dtype=torch.float64)
    check(z, ids, q.log().float().cuda(), None, 1.0, True)


def test_loss_alone_and_gradient_alone():
    z = logits_of(5, 4001, BF)
    ids, values = teacher(z, 10, 1.0, False)
    loss, d = distill(z, ids, values)
    ws = B.alloc_workspace(B.distill_topk_workspace_bytes())
    only = torch.empty_like(loss)
    B.distill_topk(z, ids, values, only, ws)
    assert torch.equal(only, loss)
    grad = torch.empty_like(d)
    B.distill_topk(z, ids, values, None, ws, d_logits=grad)
    assert torch.equal(grad, d)


def test_gradient_by_differences():
    z = logits_of(2, 40, F32, std=1.0)
    for tail in (False, True):
        ids, values = teacher(z, 6, 1.5, tail)
        _, d = distill(z, ids, values, None, 1.5, tail)
        h = 2.0 ** -6
        for j in (0, 20, int(ids[0, 0])):
            up, down = z.clone(), z.clone()
            up[:, j] += h
            down[:, j] -= h
            slope = (reference(up, ids, values, None, 1.5, tail)[0] - reference(down, ids, values, None, 1.5, tail)[0]) / (2 * h)
            assert ((d[:, j].double() - slope).abs() <= 1e-4).all()          # h^2 / 6 of third derivatives below 1


def test_many_rows_with_ids_outside():
    """more than one block looks through"""
    z = logits_of(1000, 300, BF)
    ids, values = teacher(z, 20, 1.0, True)
    check(z, ids, values, None, 1.0, True)
    ids[999, 3] = 300
    distill(z, ids, values, tail=True, status=B.E_BAD_LABEL)
    w = torch.ones(1000, device="cuda")
    w[999] = 0
    distill(z, ids, values, w, tail=True)
