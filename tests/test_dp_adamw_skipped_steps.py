"""A step that ShardedAdamW leaves out, because the norm is not finite, does not count: the moments that the next step corrects
for their start at zero have seen one update less.  On one process and on two gloo ranks, with the kernels' part in torch
(test_dp_adamw_host.py), and on the GPU."""
import os

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

import test_dp_adamw_host as H
from paper_2506_03077_b200 import dp


def updates_only(order):
    """The steps `order` unsharded, in 64 bits; their number is t."""
    p = {k: v.to(torch.bfloat16).double() for k, v in H.inputs(100).items()}
    m, v = ({n: torch.zeros_like(x) for n, x in p.items()} for _ in range(2))
    for t, s in enumerate(order, 1):
        g = {n: x.double() for n, x in H.inputs(s).items()}
        scale = min(1.0, 1.0 / (float(torch.sqrt(sum((x ** 2).sum() for x in g.values()))) + 1e-6))
        for n in p:
            x = g[n] * scale
            m[n] = 0.9 * m[n] + 0.1 * x
            v[n] = 0.95 * v[n] + 0.05 * x * x
            p[n] = (p[n] * (1 - 1e-2 * H.DECAY.get(n, 0.0)) -
                    1e-2 / (1 - 0.9 ** t) * m[n] / ((v[n] / (1 - 0.95 ** t)).sqrt() + 1e-8))
    return p


def close(got, bad):
    want = updates_only([s for s in range(3) if s != bad])
    for k in want:
        # the master copy is exact to fp32 roundings; the parameters are it, rounded once to bf16
        assert np.allclose(got[k], want[k].numpy(), rtol=2.0 ** -8 * 1.01, atol=1e-6), k


def _rank_main(rank, world, port, q, bad):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    H.host_kernels()
    got = H.run_steps(rank, world, 3, bad)
    q.put((rank, {k: v.numpy() for k, v in got.items()}))
    dist.barrier()
    dist.destroy_process_group()


@pytest.mark.parametrize("bad", [0, 1, 2])
def test_two_ranks(bad):
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    procs = [ctx.Process(target=_rank_main, args=(r, 2, 29751 + bad, q, bad)) for r in range(2)]
    for p in procs:
        p.start()
    got = dict(q.get(timeout=120) for _ in procs)
    for p in procs:
        p.join(60)
        assert p.exitcode == 0
    for k in H.SHAPES:
        assert np.array_equal(got[0][k], got[1][k])
    close(got[0], bad)


@pytest.mark.parametrize("bad", [0, 1])
def test_one_process(bad, monkeypatch):
    for name, f in (("AdamWPlan", H.HostPlan), ("grad_norm", H.host_norm), ("adamw_step", H.host_step)):
        monkeypatch.setattr(H.B, name, f)
    close({k: v.numpy() for k, v in H.run_steps(0, 1, 3, bad).items()}, bad)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_the_kernels_see_the_same_step_number(bits):
    """A bad first step, then a good one, leaves what the good one alone leaves, bit by bit."""
    def train(order):
        b = dp.GradBucket(H.SHAPES, 1, device="cuda")
        params = dp.ParamBucket(b, {k: v.to("cuda", torch.bfloat16) for k, v in H.inputs(100).items()})
        opt = dp.ShardedAdamW(params, b, b.flat, H.DECAY, bits=bits)
        for s in order:
            for k, v in H.inputs(abs(s)).items():
                b.views[k].copy_(v)
            if s < 0:
                b.views["wk"][3, 7] = float("inf")
            opt.step(**H.HYPER)
        return params.flat, opt.master, opt.m, opt.v, opt.steps
    for x, y in zip(train([-1, 2, -3, 4]), train([2, 4])):
        assert torch.equal(x, y)
