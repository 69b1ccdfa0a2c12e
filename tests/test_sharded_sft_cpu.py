"""The sharded supervised step on CPU: two gloo ranks whose kernels are stood in for by the fp64 definitions
(tests/oracle_ops.py).  What is checked is the step's logic: the global token count reaches every rank before its
loss, loss scalars and weight gradients (head and norm) add up to the unsharded result, row gradients stay with
their rank, and accumulated micro-batches are reduced once."""
import os
import sys

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from test_sharded_cpu import _free_port

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(os.path.abspath(__file__))
KW = dict(open_id=22, close_id=23, label_smoothing=0.1, z_coef=1e-2)


def _problem():
    rng = np.random.default_rng(21)
    lens = rng.integers(5, 14, size=7)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, D, V = int(cu[-1]), 8, 24
    ids = rng.integers(0, 22, size=T).astype(np.int32)
    for b in range(7):
        ids[cu[b] + 1], ids[cu[b] + 3] = 22, 23
    f = lambda *s: torch.from_numpy(rng.normal(size=s))
    return dict(cu=cu, ids=ids, x=f(T, D), res=f(T, D), W=f(V, D), w=f(D), b=f(D), logits=f(T, V))


def _steps(P, cu, ids, rows, group, ops):
    from paper_2509_06980_b200 import sharded
    rows = torch.as_tensor(rows)
    t = (torch.from_numpy(ids), torch.from_numpy(cu))
    a = sharded.sharded_sft_step(*t, logits=P["logits"][rows], group=group, ops=ops, **KW)
    b = sharded.sharded_sft_step(*t, hidden=P["x"][rows], W=P["W"], group=group, ops=ops, **KW)
    c = sharded.sharded_sft_step(*t, hidden=P["x"][rows], W=P["W"], residual=P["res"][rows], norm_weight=P["w"],
                                 norm_bias=P["b"], norm_kind=1, group=group, ops=ops, **KW)
    return a, b, c


def _worker(rank, world, port, out):
    sys.path.insert(0, ROOT)
    sys.path.insert(0, HERE)
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    import oracle_ops
    from paper_2509_06980_b200 import sharded
    P = _problem()
    plan = sharded.plan_shards(P["cu"], 1, world)[rank]
    tok = {"ids": P["ids"], "rows": np.arange(len(P["ids"]))}
    cu, t, _ = sharded.take_shard(plan, P["cu"], tok, {})
    a, b, c = _steps(P, cu, t["ids"], t["rows"], dist.group.WORLD, oracle_ops)
    # two micro-batches of this rank's responses into one grad_W, reduced with the last one
    gw, loss = torch.zeros(24, 8, dtype=torch.float64), torch.zeros(4, dtype=torch.float64)
    parts = [plan[:1], plan[1:]]
    for k, part in enumerate(parts):
        cu_k, t_k, _ = sharded.take_shard(part, P["cu"], tok, {})
        o = sharded.sharded_sft_step(torch.from_numpy(t_k["ids"]), torch.from_numpy(cu_k), hidden=P["x"][torch.as_tensor(t_k["rows"])],
                                     W=P["W"], grad_W=gw, accumulate_grad_W=k > 0, reduce_grads=k == 1,
                                     n_global=a["n_global"], group=dist.group.WORLD, ops=oracle_ops, **KW)
        loss += o["loss"]
    n = lambda d: {k: v.numpy() for k, v in d.items()}
    out.put((rank, t["rows"], n(a), n(b), n(c), gw.numpy(), loss.numpy()))
    dist.barrier()
    dist.destroy_process_group()


def test_two_ranks_add_up_to_the_unsharded_step():
    import oracle_ops
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
    whole = _steps(P, P["cu"], P["ids"], np.arange(len(P["ids"])), None, oracle_ops)
    n = whole[0]["n_global"].item()
    assert sum(g[2]["n_local"].item() for g in got) == n and 0 < n < len(P["ids"])
    for _, rows, a, b, c, gw, loss in got:
        for mine, ref in zip((a, b, c), whole):
            assert mine["n_global"].item() == n and set(mine) == set(ref)
            for k, v in ref.items():
                if k in ("n_local", "n_global"):
                    continue
                want = v.numpy()
                if k in ("mask", "logp", "lse", "grad_logits", "grad_hidden"):
                    want = want[rows]                                    # row results stay with their rank
                assert np.allclose(mine[k], want, rtol=1e-11, atol=1e-15, equal_nan=True), k
        assert np.allclose(gw, whole[1]["grad_W"].numpy(), rtol=1e-11, atol=1e-15)
        assert np.allclose(loss, whole[1]["loss"].numpy(), rtol=1e-12)
    assert {"grad_norm_weight", "grad_norm_bias"} <= set(got[0][4]) and "grad_norm_weight" not in got[0][3]


def test_arguments_that_do_not_go_together():
    import oracle_ops
    from paper_2509_06980_b200 import sharded
    P = _problem()
    t = (torch.from_numpy(P["ids"]), torch.from_numpy(P["cu"]))
    for kw in (dict(), dict(logits=P["logits"], hidden=P["x"], W=P["W"]), dict(logits=P["logits"], norm_weight=P["w"]),
               dict(hidden=P["x"], W=P["W"], residual=P["res"])):
        with pytest.raises(ValueError):
            sharded.sharded_sft_step(*t, ops=oracle_ops, **KW, **kw)
