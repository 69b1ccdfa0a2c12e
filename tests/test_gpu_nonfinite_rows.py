"""A NaN among logits of which its warp, column tile or split of the vocabulary holds no finite one: the row has no
log-prob (NaN), no gradient and raises the status, in every call that takes logits or a head."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _tokens(T, V, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    seq = torch.zeros(T, dtype=torch.int32, device=DEV)
    adv = torch.ones(1, device=DEV)
    old = torch.zeros(T, device=DEV)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    return g, ids, seq, adv, old, mask


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T", [12, 700])
@pytest.mark.parametrize("V", [1000, 2056, 8192, 50304, 151936])
def test_rows_of_logits(T, V, dt):
    b = gc.binding()
    nan, inf = float("nan"), float("inf")
    if T * V > 1 << 26:
        T = 520
    g, ids, seq, adv, old, mask = _tokens(T, V, V)
    z = torch.randn(T, V, generator=g, device=DEV).to(dt)
    ids[:5] = V // 2
    z[0] = nan
    z[0, V // 2] = 1.0                       # nothing but the target is a number
    z[1] = -inf
    z[1, V // 2], z[1, V - 1] = 0.5, nan     # a masked vocabulary with one NaN
    z[2] = -inf
    z[2, V // 2], z[2, 3] = 0.5, nan
    z[3, V // 2 + 8:] = nan
    z[4] = -inf
    z[4, V // 2], z[4, 0] = 0.5, 0.25        # a masked vocabulary, sound
    gone = torch.zeros(T, dtype=torch.bool, device=DEV)
    gone[:4] = True
    calls = [lambda st: b.rlf_grpo_logp_loss_fwd_bwd(z, ids, seq, adv, old, old, mask, 0.2, 0.01, dev_status=st),
             lambda st: b.rlf_grpo_logp_loss_fwd_bwd_obj(z, ids, seq, adv, old, old, mask, 0.2, 0.2, 0.01, aggregation=1, dev_status=st)]
    if dt == BF:
        calls.append(lambda st: b.rlf_grpo_logp_loss_fwd_bwd_skip_masked(z, ids, seq, adv, old, old, mask, 0.2, 0.01, dev_status=st))
    for k, call in enumerate(calls):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        logp, loss, grad = call(st)[:3]
        assert st.item() == b.DEV_NONFINITE, k
        assert torch.equal(torch.isnan(logp), gone), (k, logp[:6])
        assert torch.isfinite(loss).all() and torch.isfinite(grad).all() and not grad[gone].any(), k
    if dt == BF:
        for want in (True, False):
            st = torch.zeros(1, dtype=torch.int32, device=DEV)
            logp, ent = b.rlf_logp_entropy_fwd(z, ids, want_entropy=want, dev_status=st)
            assert st.item() == b.DEV_NONFINITE and torch.equal(torch.isnan(logp), gone), (want, logp[:6])
            assert ent is None or torch.isnan(ent[gone]).all()


@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("V,first,last", [(1032, 1024, 1032), (1032, 256, 512), (1032, 0, 256), (264, 256, 264), (20008, 19968, 20008)])
def test_nan_rows_of_a_head(T, V, first, last):
    b = gc.binding()
    g, ids, seq, adv, old, mask = _tokens(T, V, 7)
    H = torch.randn(T, 64, generator=g, device=DEV).to(BF)
    W = (0.25 * torch.randn(V, 64, generator=g, device=DEV)).to(BF)
    W[first:last] = float("nan")
    ids.clamp_(max=first - 1) if first else ids.clamp_(min=last)
    for agg in (0, 1):
        for row_reference in (1, 0):
            st = torch.zeros(1, dtype=torch.int32, device=DEV)
            b.tune_lmhead_backward(row_reference, 1)
            try:
                logp, loss = b.rlf_fused_lmhead_grpo_obj(H, W, ids, seq, adv, old, old, mask, 0.2, 0.2, 0.01, aggregation=agg,
                                                         dev_status=st)[:2]
            finally:
                b.tune_lmhead_backward(1, 1)
            assert st.item() == b.DEV_NONFINITE and torch.isnan(logp).all() and torch.isfinite(loss).all(), (agg, row_reference)
    for want in (True, False):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        logp, ent = b.rlf_fused_lmhead_logp_entropy(H, W, ids, want_entropy=want, dev_status=st)
        assert st.item() == b.DEV_NONFINITE and torch.isnan(logp).all() and (ent is None or torch.isnan(ent).all()), want
