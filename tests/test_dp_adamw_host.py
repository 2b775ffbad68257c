"""Sharded AdamW on CPU: the layout of the shards' pieces, and with two gloo ranks the exchange around the step -- one norm
over all ranks, every rank its slice, the parameters gathered.  The kernels' part is a few lines of torch here; the kernels
themselves are tested on the GPU."""
import os
import sys

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
from paper_2506_03077_b200 import binding as B  # noqa: E402
from paper_2506_03077_b200 import dp  # noqa: E402

SHAPES = {"g1": (40,), "wq": (48, 40), "bq": (48,), "wk": (16, 40), "w_down": (40, 100)}
DECAY = {"wq": 0.1, "wk": 0.1, "w_down": 0.1}
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)


@pytest.mark.parametrize("world", [1, 2, 3, 8, 64])
def test_pieces_tile_the_tensors_and_start_on_block_boundaries(world):
    b = dp.GradBucket(SHAPES, world, device="cpu")
    owned = {k: 0 for k in SHAPES}
    for r in range(world):
        end = 0
        for name, a, e in dp.shard_slices(b, r):
            assert a % dp.ALIGN_ELEMS == 0 and end <= a < e <= b.shard_elems
            end = e
            owned[name] += e - a
            lo = b.shard_range(r)[0]
            o, n = b.table[name]
            assert o <= lo + a and lo + e <= o + n
    assert owned == {k: int(np.prod(s)) for k, s in SHAPES.items()}


class HostPlan:
    def __init__(self, tensors):
        self.tensors = tensors


def host_norm(plan, max_norm, norm, scale, workspace, **kw):
    n = torch.sqrt(sum((t["grad"].double() ** 2).sum() for t in plan.tensors)).float()
    norm.fill_(n)
    scale.copy_((max_norm / (norm + 1e-6)).clamp(max=1.0) + (norm - norm))


def host_step(plan, lr, beta1, beta2, eps, step, grad_scale=None, **kw):
    s, k = float(grad_scale), int(step)
    if not np.isfinite(s):
        return
    for t in plan.tensors:
        g = t["grad"] * s
        t["m"].mul_(beta1).add_(g, alpha=1 - beta1)
        t["v"].mul_(beta2).add_(g * g, alpha=1 - beta2)
        p = t.get("master", t["param"])
        p.mul_(1 - lr * t["weight_decay"])
        p.sub_(lr / (1 - beta1 ** k) * t["m"] / ((t["v"] / (1 - beta2 ** k)).sqrt() + eps))
        if p is not t["param"]:
            t["param"].copy_(p)


def host_kernels():
    B.AdamWPlan, B.grad_norm, B.adamw_step = HostPlan, host_norm, host_step


def inputs(step, shapes=SHAPES):
    g = torch.Generator().manual_seed(step)
    return {k: torch.randn(s, generator=g) for k, s in shapes.items()}


def whole(steps, bad=None, shapes=SHAPES):
    """The same steps unsharded, in 64 bits."""
    p = {k: v.to(torch.bfloat16).double() for k, v in inputs(100, shapes).items()}
    m, v, k = ({n: torch.zeros_like(x) for n, x in p.items()} for _ in range(2)), None, 0
    m, v = m
    for s in range(steps):
        g = {n: x.double() for n, x in inputs(s, shapes).items()}
        k += 1
        if s == bad:
            continue
        scale = min(1.0, 1.0 / (float(torch.sqrt(sum((x ** 2).sum() for x in g.values()))) + 1e-6))
        for n in p:
            x = g[n] * scale
            m[n] = 0.9 * m[n] + 0.1 * x
            v[n] = 0.95 * v[n] + 0.05 * x * x
            p[n] = p[n] * (1 - 1e-2 * DECAY.get(n, 0.0)) - 1e-2 / (1 - 0.9 ** k) * m[n] / ((v[n] / (1 - 0.95 ** k)).sqrt() + 1e-8)
    return p


def run_steps(rank, world, steps, bad=None, shapes=SHAPES):
    b = dp.GradBucket(shapes, world, device="cpu")
    params = dp.ParamBucket(b, {k: v.to(torch.bfloat16) for k, v in inputs(100, shapes).items()})
    shard = torch.zeros(b.shard_elems)
    opt = dp.ShardedAdamW(params, b, shard, {k: v for k, v in DECAY.items() if k in shapes}, bits=32)
    for s in range(steps):
        for k, v in inputs(s, shapes).items():
            b.views[k].copy_(v / world)
        if s == bad and rank == world - 1:
            b.views["w_down"][0, 0] = float("nan")
        if world > 1:
            dp.reduce_scatter_sum(b.flat, shard)
        else:
            shard.copy_(b.flat)
        opt.step(**HYPER)
    return {k: v.float().clone() for k, v in params.views.items()}


def _rank_main(rank, world, port, q, bad, shapes):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    host_kernels()
    got = run_steps(rank, world, 3, bad, shapes)
    q.put((rank, {k: v.numpy() for k, v in got.items()}))
    dist.barrier()
    dist.destroy_process_group()


@pytest.mark.parametrize("bad,shapes", [(None, SHAPES), (1, SHAPES), (None, {"g1": (40,)})], ids=["three", "bad", "empty"])
def test_two_ranks_step_as_one(bad, shapes):
    """bad: a gradient that is not a number on one rank leaves that step out on both.  empty: the second rank's shard holds
    padding only."""
    world, port = 2, 29731 + (bad or 0) + 2 * (shapes is not SHAPES)
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    procs = [ctx.Process(target=_rank_main, args=(r, world, port, q, bad, shapes)) for r in range(world)]
    for p in procs:
        p.start()
    got = dict(q.get(timeout=120) for _ in procs)
    for p in procs:
        p.join(60)
        assert p.exitcode == 0
    want = whole(3, bad, shapes)
    for k in shapes:
        assert np.array_equal(got[0][k], got[1][k])
        # the master copy is exact to fp32 roundings; the parameters are it, rounded once to bf16
        assert np.allclose(got[0][k], want[k].numpy(), rtol=2.0 ** -8 * 1.01, atol=1e-6)


def test_sizes_must_match():
    b = dp.GradBucket(SHAPES, 2, device="cpu")
    params = dp.ParamBucket(b, inputs(0))
    with pytest.raises(ValueError):
        dp.ShardedAdamW(params, b, torch.zeros(b.shard_elems), DECAY)                 # one process, laid out for two
    with pytest.raises(ValueError):
        dp.ShardedAdamW(params, b, torch.zeros(8), DECAY, rank=0, world=2)
    with pytest.raises(ValueError):
        dp.ShardedAdamW(params, b, torch.zeros(b.shard_elems), DECAY, bits=4, rank=0, world=2)
    with pytest.raises(ValueError):
        dp.ShardedAdamW(params, b, torch.zeros(b.shard_elems), {"wqq": 0.1}, rank=0, world=2)
