"""Micro-batches of the supervised step with the kernels: the head's and the norm's weight gradients accumulate in the
caller's buffers."""
import numpy as np
import pytest
import torch

from paper_2509_06980_b200 import sharded
import gpu_common as gc
from test_gpu_sft_step import DEV, _batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_micro_batches_add_up_to_the_whole_batch(layer):
    """The parts' sums are those of the whole batch but for the order of additions and, in the head's two products, the
    split's own roundings to bf16 (2^-8 each of entries that enter the sums with either sign): 2^-7 of the largest value."""
    b = gc.binding()
    spec, tok, ids, cu, x, res, W, w, bias = _batch()
    kw = dict(W=W, norm_weight=w, norm_bias=bias if layer else None, norm_kind=b.NORM_LAYER if layer else b.NORM_RMS,
              label_smoothing=0.1, z_coef=1e-4)
    whole = sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, hidden=x, residual=res, **kw)
    names = ["grad_W", "grad_norm_weight"] + (["grad_norm_bias"] if layer else [])
    bufs = {k: torch.full_like(whole[k], 7.0) for k in names}
    n = len(tok.cu_seqlens) - 1
    loss = 0.0
    for k, part in enumerate((np.arange(1), np.arange(1, n - 2), np.arange(n - 2, n))):
        cu_k, t_k, _ = sharded.take_shard(part, tok.cu_seqlens, {"ids": tok.ids, "rows": np.arange(len(tok.ids))}, {})
        rows = torch.from_numpy(t_k["rows"]).to(DEV)
        o = sharded.sharded_sft_step(torch.from_numpy(t_k["ids"]).to(DEV), torch.from_numpy(cu_k).to(DEV), spec.open_id,
                                     spec.close_id, hidden=x[rows], residual=res[rows], n_global=whole["n_global"],
                                     accumulate_grad_W=k > 0, **bufs, **kw)
        loss = loss + o["loss"]
        assert all(o[name] is buf for name, buf in bufs.items())
    assert torch.allclose(loss, whole["loss"], rtol=1e-6)
    for name, buf in bufs.items():
        assert (buf - whole[name]).abs().max() <= 2.0 ** -7 * whole[name].abs().max(), name
