"""Data-parallel streamed backward: one process per GPU, each on its own sequences, and ONE exchange per layer.

The paper's distributed setting (Sec. 3.3 and App. A.3, "Distributed StreamBP", gradient communication
design) keeps the sequence-partitioned accumulation local to a rank: g_W is summed over the partitions D of that rank's sequences first, and only the
finished per-layer sum crosses the interconnect -- one gradient reduce-scatter (or all-reduce) per layer after
its chunk loop, instead of one per partition.  This module is the plumbing for that:

  * GradBucket  -- every fp32 weight-gradient tensor of a layer is a view into one flat buffer, each view
                   256-byte aligned (the C ABI wants 16), the total padded so that it splits evenly over the
                   ranks.  The library accumulates into the views; the exchange sees one contiguous tensor.
  * reduce_scatter_sum / all_reduce_sum -- torch.distributed on whatever backend the group has (NCCL over
                   NVLink / NVSwitch on GPUs; gloo on CPU, where reduce-scatter is an all-reduce plus a slice).
  * DataParallelLayerBackward -- layer backward on the compute stream, then the bucket's reduce-scatter on a
                   communication stream, so that the exchange of layer l overlaps the chunk loop of layer l-1.

Nothing here computes a gradient: the arithmetic is the library's (streambp_layer_backward) and NCCL's sum.
No kernel of the library reads another GPU's memory, and no TMA multicast is used anywhere.
"""
from __future__ import annotations

from typing import Dict, List, Tuple

import torch
import torch.distributed as dist

ALIGN_ELEMS = 64          # 256 bytes of fp32


def bucket_layout(shapes: Dict[str, Tuple[int, ...]], world: int) -> Tuple[Dict[str, Tuple[int, int]], int]:
    """Offsets (in fp32 elements) of every tensor inside the flat bucket and the padded total.

    Tensors are laid out in the order of `shapes`, each starting on a 256-byte boundary; the total is rounded
    up to a multiple of world * ALIGN_ELEMS so that every rank's shard has the same size and alignment."""
    if world < 1:
        raise ValueError("world must be >= 1")
    off, table = 0, {}
    for name, shp in shapes.items():
        n = 1
        for s in shp:
            n *= int(s)
        off = (off + ALIGN_ELEMS - 1) // ALIGN_ELEMS * ALIGN_ELEMS
        table[name] = (off, n)
        off += n
    unit = world * ALIGN_ELEMS
    total = (off + unit - 1) // unit * unit
    return table, total


class GradBucket:
    """Flat fp32 gradient storage of one layer with named views."""

    def __init__(self, shapes: Dict[str, Tuple[int, ...]], world: int, device="cuda"):
        self.shapes, self.world = dict(shapes), world
        self.table, self.total = bucket_layout(shapes, world)
        self.flat = torch.zeros(self.total, dtype=torch.float32, device=device)
        self.views = {k: self.flat[o:o + n].view(self.shapes[k]) for k, (o, n) in self.table.items()}
        self.shard_elems = self.total // world

    def shard_range(self, rank: int) -> Tuple[int, int]:
        return rank * self.shard_elems, (rank + 1) * self.shard_elems

    def owner_slices(self, rank: int) -> Dict[str, Tuple[int, int]]:
        """For each tensor, the [begin, end) range of its flattened elements that rank's shard holds."""
        lo, hi = self.shard_range(rank)
        out = {}
        for k, (o, n) in self.table.items():
            a, b = max(lo, o), min(hi, o + n)
            if a < b:
                out[k] = (a - o, b - o)
        return out


def reduce_scatter_sum(flat: torch.Tensor, shard: torch.Tensor, group=None) -> None:
    """shard <- this rank's slice of the element-wise sum of `flat` over the group."""
    world = dist.get_world_size(group)
    rank = dist.get_rank(group)
    n = flat.numel() // world
    assert flat.numel() == n * world and shard.numel() == n
    if dist.get_backend(group) == "nccl":
        dist.reduce_scatter_tensor(shard, flat, op=dist.ReduceOp.SUM, group=group)
    else:   # gloo has no reduce-scatter: same result through an all-reduce
        tmp = flat.clone()
        dist.all_reduce(tmp, op=dist.ReduceOp.SUM, group=group)
        shard.copy_(tmp[rank * n:(rank + 1) * n])


def all_reduce_sum(flat: torch.Tensor, group=None) -> None:
    dist.all_reduce(flat, op=dist.ReduceOp.SUM, group=group)


class DataParallelLayerBackward:
    """streambp_layer_backward on this rank's sequence, then one reduce-scatter of the layer's gradient bucket.

    step() enqueues the backward on the compute stream and the exchange on a communication stream that waits
    for it; the caller goes on to the next layer (or the next micro-batch with accumulate=True, in which case
    it passes exchange=False until the last one) and calls wait() before reading `shard`."""

    def __init__(self, cfg, weights, T: int, chunk: int, group=None, device="cuda"):
        from . import binding as B
        self.B, self.cfg, self.weights, self.chunk, self.group = B, cfg, weights, chunk, group
        self.world = dist.get_world_size(group) if dist.is_initialized() else 1
        self.rank = dist.get_rank(group) if dist.is_initialized() else 0
        self.bucket = GradBucket(B.layer_grad_shapes(cfg), self.world, device)
        self.shard = torch.zeros(self.bucket.shard_elems, dtype=torch.float32, device=device)
        self.ws = B.alloc_workspace(B.layer_workspace_bytes(cfg, T, chunk), device)
        self.comm_stream = torch.cuda.Stream(device=device)
        self.computed = torch.cuda.Event()
        self.exchanged = torch.cuda.Event()

    def step(self, X, dY, dX, accumulate: bool = False, exchange: bool = True, stream=None) -> None:
        st = stream if stream is not None else torch.cuda.current_stream()
        st.wait_event(self.exchanged)      # a previous exchange may still be reading the bucket (no-op before the first)
        self.B.layer_backward(self.cfg, self.weights, X, dY, self.chunk, self.bucket.views, dX, self.ws,
                              accumulate=accumulate, stream=st)
        if not exchange:
            return
        self.computed.record(st)
        self.comm_stream.wait_event(self.computed)
        with torch.cuda.stream(self.comm_stream):
            if self.world > 1:
                reduce_scatter_sum(self.bucket.flat, self.shard, self.group)
            else:
                self.shard.copy_(self.bucket.flat)
            self.exchanged.record(self.comm_stream)

    def wait(self, stream=None) -> None:
        st = stream if stream is not None else torch.cuda.current_stream()
        st.wait_event(self.exchanged)


def gather_full_gradients(bucket: GradBucket, shard: torch.Tensor, group=None) -> Dict[str, torch.Tensor]:
    """All ranks' shards reassembled into named tensors (for tests and for optimizers that want full tensors)."""
    world = dist.get_world_size(group) if dist.is_initialized() else 1
    if world > 1:
        parts: List[torch.Tensor] = [torch.empty_like(shard) for _ in range(world)]
        dist.all_gather(parts, shard, group=group)
        flat = torch.cat(parts)
    else:
        flat = shard
    return {k: flat[o:o + n].view(bucket.shapes[k]).clone() for k, (o, n) in bucket.table.items()}


class ParamBucket:
    """Flat parameters of one layer in the layout of its GradBucket (storage dtype), with named views: what the backward
    reads as weights, and what a sharded optimizer writes one slice of per rank."""

    def __init__(self, grads: GradBucket, values: Dict[str, torch.Tensor]):
        dtype = next(iter(values.values())).dtype
        self.flat = torch.zeros(grads.total, dtype=dtype, device=grads.flat.device)
        self.views = {k: self.flat[o:o + n].view(grads.shapes[k]) for k, (o, n) in grads.table.items()}
        for k, v in self.views.items():
            v.copy_(values[k])


def shard_slices(bucket: GradBucket, rank: int) -> List[Tuple[str, int, int]]:
    """(name, begin, end) of every piece of a tensor inside a rank's shard, as offsets into the shard.  Tensors and shards
    start on ALIGN_ELEMS boundaries, so every piece does too: aligned for the kernels, and a whole number of blocks of
    8-bit moments before it."""
    lo, _ = bucket.shard_range(rank)
    out = []
    for name, (a, b) in bucket.owner_slices(rank).items():
        at = bucket.table[name][0] + a - lo
        out.append((name, at, at + b - a))
    return out


class ShardedAdamW:
    """One AdamW step of a layer's parameters, each rank on its shard of the summed gradients: the moments and the fp32
    master copy exist once over all ranks.  `shard` is what DataParallelLayerBackward.exchange leaves (wait() first).
    step() clips by the norm over the whole layer (an all-reduce of one number), updates this rank's slice on the library's
    kernels and gathers the rounded parameters of all ranks.  A norm that is not finite leaves every rank's slice as it was, and
    the step does not count (`steps`, on the device: the updates so far).  Over several ranks a norm beyond
    fp32's range is such a norm.

    weight_decay: per tensor name (missing: 0).  bits: 32, or 8 for moments in blocks of 32 e4m3 codes."""

    def __init__(self, params: ParamBucket, grads: GradBucket, shard: torch.Tensor, weight_decay: Dict[str, float],
                 bits: int = 8, group=None, rank: int = None, world: int = None):
        from . import binding as B
        if bits not in (8, 32):
            raise ValueError("moments have 8 or 32 bits")
        ready = dist.is_initialized()
        self.rank = rank if rank is not None else (dist.get_rank(group) if ready else 0)
        self.world = world if world is not None else (dist.get_world_size(group) if ready else 1)
        if grads.world != self.world or shard.numel() != grads.shard_elems:
            raise ValueError(f"the bucket is laid out for {grads.world} ranks, the group has {self.world}")
        if not weight_decay.keys() <= grads.table.keys():
            raise ValueError(f"no such tensors: {sorted(weight_decay.keys() - grads.table.keys())}")
        self.B, self.params, self.shard, self.group = B, params, shard, group
        lo, hi = grads.shard_range(self.rank)
        self.param = params.flat[lo:hi]
        f32, dev, n = self.param.dtype == torch.float32, shard.device, hi - lo
        self.master = None if f32 else self.param.float()
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8 if bits == 8 else torch.float32, device=dev) for _ in range(2))
        self.scales = [torch.ones(n // B.MX8_BLOCK, dtype=torch.uint8, device=dev) for _ in range(2)] if bits == 8 else None
        tensors = []
        for name, a, b in shard_slices(grads, self.rank):
            t = {"param": self.param[a:b], "grad": shard[a:b], "m": self.m[a:b], "v": self.v[a:b],
                 "weight_decay": weight_decay.get(name, 0.0)}
            if self.master is not None:
                t["master"] = self.master[a:b]
            if bits == 8:
                s = slice(a // B.MX8_BLOCK, (b + B.MX8_BLOCK - 1) // B.MX8_BLOCK)
                t["m_scale"], t["v_scale"] = self.scales[0][s], self.scales[1][s]
            tensors.append(t)
        self.plan = B.AdamWPlan(tensors) if tensors else None      # a short last shard may hold padding only
        self.norm, self.scale = torch.zeros(1, device=dev), torch.ones(1, device=dev)
        self.steps = torch.zeros(1, dtype=torch.int64, device=dev)
        self.ws = B.alloc_workspace(B.grad_norm_workspace_bytes(), dev)

    def step(self, lr: float, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, max_norm: float = 1.0) -> None:
        """On the current stream."""
        if self.plan is not None:
            self.B.grad_norm(self.plan, max_norm, self.norm, self.scale, self.ws)
        else:
            self.norm.zero_()
        if self.world > 1:
            total = self.norm.double().square_()
            dist.all_reduce(total, group=self.group)
            self.norm.copy_(total.sqrt_())
            # what grad_norm writes for one rank; norm - norm is NaN where the norm is not finite
            self.scale.copy_((max_norm / (self.norm + 1e-6)).clamp_(max=1.0) + (self.norm - self.norm))
        self.steps += torch.isfinite(self.scale)          # on the device: the host does not wait for the norm
        if self.plan is not None:
            self.B.adamw_step(self.plan, lr, beta1, beta2, eps, self.steps, grad_scale=self.scale)
        if self.world > 1:
            if dist.get_backend(self.group) == "nccl":
                dist.all_gather_into_tensor(self.params.flat, self.param.clone(), group=self.group)
            else:
                parts = [torch.empty_like(self.param) for _ in range(self.world)]
                dist.all_gather(parts, self.param, group=self.group)
                self.params.flat.copy_(torch.cat(parts))
