"""Micro-batches of the sharded supervised step, norm included, on two gloo ranks with the fp64 definitions as
kernels: the head's and the norm's weight gradients accumulate over a rank's micro-batches and are reduced once."""
import os
import sys

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from test_sharded_cpu import _free_port
from test_sharded_sft_cpu import HERE, KW, ROOT, _problem


class Ops:
    """tests/oracle_ops.py with a norm backward that takes buffers."""

    def __getattr__(self, name):
        import oracle_ops
        return getattr(oracle_ops, name)

    def rlf_norm_bwd(self, *a, grad_weight=None, grad_bias=None, accumulate=False, **kw):
        import oracle_ops
        gx, gw, gb = oracle_ops.rlf_norm_bwd(*a, **kw)
        out = []
        for g, buf in ((gw, grad_weight), (gb, grad_bias)):
            if buf is not None:
                buf.copy_(buf + g if accumulate else g)
            out.append(g if buf is None else buf)
        return (gx, *out)


def _norm(P, rows, bias):
    rows = torch.as_tensor(rows)
    kw = dict(hidden=P["x"][rows], W=P["W"], residual=P["res"][rows], norm_weight=P["w"], norm_kind=1 if bias else 0)
    return dict(kw, norm_bias=P["b"]) if bias else kw


def _worker(rank, world, port, out):
    sys.path.insert(0, ROOT)
    sys.path.insert(0, HERE)
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from paper_2509_06980_b200 import sharded
    P = _problem()
    plan = sharded.plan_shards(P["cu"], 1, world)[rank]
    tok = {"ids": P["ids"], "rows": np.arange(len(P["ids"]))}
    n = torch.zeros(1, dtype=torch.int64)
    for part in (plan[:1], plan[1:]):
        cu, t, _ = sharded.take_shard(part, P["cu"], tok, {})
        n += sharded.count_phase(torch.from_numpy(t["ids"]), torch.from_numpy(cu), KW["open_id"], KW["close_id"], Ops())[2]
    dist.all_reduce(n)
    got = []
    for bias in (True, False):
        bufs = dict(grad_W=torch.full((24, 8), 9.0, dtype=torch.float64), grad_norm_weight=torch.full((8,), 9.0, dtype=torch.float64))
        if bias:
            bufs["grad_norm_bias"] = torch.full((8,), 9.0, dtype=torch.float64)
        for k, part in enumerate((plan[:1], plan[1:2], plan[2:])):
            cu, t, _ = sharded.take_shard(part, P["cu"], tok, {})
            o = sharded.sharded_sft_step(torch.from_numpy(t["ids"]), torch.from_numpy(cu), **_norm(P, t["rows"], bias), **bufs,
                                         accumulate_grad_W=k > 0, reduce_grads=k == 2, n_global=n, group=dist.group.WORLD,
                                         ops=Ops(), **KW)
            assert all(o[name] is buf for name, buf in bufs.items())
        got.append({name: buf.numpy() for name, buf in bufs.items()})
    out.put((rank, got))
    dist.barrier()
    dist.destroy_process_group()


def test_weight_gradients_of_micro_batches_are_those_of_the_whole_batch():
    from paper_2509_06980_b200 import sharded
    ctx = mp.get_context("spawn")
    out = ctx.SimpleQueue()
    port = _free_port()
    procs = [ctx.Process(target=_worker, args=(r, 2, port, out)) for r in range(2)]
    for p in procs:
        p.start()
    got = [out.get() for _ in range(2)]
    for p in procs:
        p.join(180)
        assert p.exitcode == 0
    P = _problem()
    for k, bias in enumerate((True, False)):
        whole = sharded.sharded_sft_step(torch.from_numpy(P["ids"]), torch.from_numpy(P["cu"]),
                                         **_norm(P, np.arange(len(P["ids"])), bias), ops=Ops(), **KW)
        for _, g in got:
            for name, v in g[k].items():
                assert np.allclose(v, whole[name].numpy(), rtol=1e-11, atol=1e-15), (bias, name)


def test_buffers_that_do_not_belong():
    from paper_2509_06980_b200 import sharded
    P = _problem()
    t = (torch.from_numpy(P["ids"]), torch.from_numpy(P["cu"]))
    buf = torch.zeros(8, dtype=torch.float64)
    gw = torch.zeros(24, 8, dtype=torch.float64)
    for kw in (dict(hidden=P["x"], W=P["W"], grad_norm_weight=buf), dict(logits=P["logits"], grad_norm_weight=buf),
               dict(hidden=P["x"], W=P["W"], norm_weight=P["w"], grad_norm_bias=buf),
               dict(hidden=P["x"], W=P["W"], norm_weight=P["w"], norm_bias=P["b"], grad_norm_weight=buf, grad_W=gw, accumulate_grad_W=True)):
        with pytest.raises(ValueError):
            sharded.sharded_sft_step(*t, ops=Ops(), **KW, **kw)
