"""Pins of the fp64 definitions in oracle/operators64.py: closed forms, invariants, central differences and
fp64 autograd, so that the GPU tests compare against something that is itself checked."""
import numpy as np
import pytest
import torch

from oracle import operators64 as o64
from oracle import rlf_oracle as orc


def _ce_autograd(z, ids, mask, eps, zc, n):
    zt = torch.tensor(z, dtype=torch.float64, requires_grad=True)
    lp = torch.log_softmax(zt, dim=1)
    l = torch.logsumexp(zt, dim=1)
    at = torch.arange(len(ids))
    term = (1 - eps) * -lp[at, torch.as_tensor(ids)] + eps * -lp.mean(dim=1) + zc * l * l
    loss = (term * torch.tensor(mask, dtype=torch.float64)).sum() / n
    loss.backward()
    return loss.item(), zt.grad.numpy()


@pytest.mark.parametrize("eps,zc", [(0.0, 0.0), (0.1, 0.0), (0.0, 1e-2), (0.2, 1e-3)])
def test_cross_entropy_against_autograd_and_differences(eps, zc):
    rng = np.random.default_rng(3)
    T, V = 7, 13
    z = rng.normal(size=(T, V)) * 3
    ids = rng.integers(0, V, T)
    mask = np.array([1, 0, 1, 1, 0, 1, 1])
    r = o64.cross_entropy(z, ids, mask, eps, zc)
    want, grad = _ce_autograd(z, ids, mask, eps, zc, 5)
    assert abs(r["loss"][0] - want) < 1e-12 and np.abs(r["grad"] - grad).max() < 1e-13
    assert not r["grad"][mask == 0].any() and np.isnan(r["logp"][mask == 0]).all()
    # rows of the gradient sum to 2 zeta lse / N: the softmax part sums to one, the target part to one
    assert np.allclose(r["grad"].sum(axis=1)[mask == 1], 2 * zc * r["lse"][mask == 1] / 5, atol=1e-14)
    h = 1e-5
    for t, v in ((0, 3), (2, int(ids[2])), (6, 0)):
        zp, zm = z.copy(), z.copy()
        zp[t, v] += h
        zm[t, v] -= h
        d = (o64.cross_entropy(zp, ids, mask, eps, zc)["loss"][0] - o64.cross_entropy(zm, ids, mask, eps, zc)["loss"][0]) / (2 * h)
        assert abs(d - r["grad"][t, v]) < 1e-8


def test_cross_entropy_closed_forms_and_neutralised_rows():
    V = 50
    r = o64.cross_entropy(np.full((2, V), 7.0), [0, 49], smoothing=0.3)
    assert np.allclose(r["logp"], -np.log(V)) and np.allclose(r["loss"][:3], np.log(V))
    # a bad target and a non-finite row lose their weight but stay in the denominator; the rest is unchanged
    z = np.random.default_rng(0).normal(size=(4, V))
    z[2, 5] = np.nan
    a = o64.cross_entropy(z, [1, -100, 3, V - 1])
    assert a["live"].tolist() == [True, False, False, True] and a["n"] == 4 and not a["grad"][1:3].any()
    # the two-argument objective reduces to the GRPO oracle's log-prob
    lp, _ = orc.logp_entropy(z[[0, 3]], np.array([1, V - 1], np.int32))
    assert np.abs(a["logp"][[0, 3]] - lp).max() < 1e-12
    # micro-batches against a common denominator add up
    b = o64.cross_entropy(z[:2], [1, -100], denom=4)["loss"] + o64.cross_entropy(z[2:], [3, V - 1], denom=4)["loss"]
    assert np.allclose(a["loss"], b, rtol=1e-14)


def test_fused_cross_entropy_is_the_chain_rule_and_smoothing_is_rank_one():
    rng = np.random.default_rng(5)
    T, D, V = 6, 8, 21
    H, W = rng.normal(size=(T, D)), rng.normal(size=(V, D))
    ids, mask = rng.integers(0, V, T), np.array([1, 1, 0, 1, 1, 1])
    r = o64.fused_cross_entropy(H, W, ids, mask, 0.1, 1e-3)
    Ht, Wt = (torch.tensor(a, requires_grad=True) for a in (H, W))
    lp = torch.log_softmax(Ht @ Wt.t(), dim=1)
    l = torch.logsumexp(Ht @ Wt.t(), dim=1)
    term = 0.9 * -lp[torch.arange(T), torch.as_tensor(ids)] - 0.1 * lp.mean(dim=1) + 1e-3 * l * l
    ((term * torch.tensor(mask, dtype=torch.float64)).sum() / 5).backward()
    assert np.abs(r["grad_hidden"] - Ht.grad.numpy()).max() < 1e-13
    assert np.abs(r["grad_W"] - Wt.grad.numpy()).max() < 1e-13
    # without the uniform part, and that part added as one row times one column
    z = H @ W.T
    p = np.exp(z - r["lse"][:, None])
    c = np.where(mask != 0, 0.2, 0.0)
    d = np.where(mask[:, None] != 0, c[:, None] * (1 + 2e-3 * r["lse"][:, None]) * p, 0.0)
    d[np.arange(T), ids] -= 0.9 * c
    assert np.allclose(d @ W - np.outer(c * 0.1 / V, W.sum(axis=0)), r["grad_hidden"], atol=1e-13)
    assert np.allclose(d.T @ H - 0.1 / V * (c[:, None] * H).sum(axis=0), r["grad_W"], atol=1e-13)


@pytest.mark.parametrize("layer", [False, True])
def test_norm_against_autograd(layer):
    rng = np.random.default_rng(7)
    T, D = 5, 11
    x, res, w, b, dy, skip = (rng.normal(size=s) for s in ((T, D), (T, D), D, D, (T, D), (T, D)))
    y, h, mu, r = o64.norm(x, w, b, res, layer, 1e-3)
    dx, dw, db = o64.norm_grad(dy, h, w, mu, r, layer, skip)
    xt, wt, bt = (torch.tensor(a, requires_grad=True) for a in (x, w, b))
    ht = xt + torch.tensor(res)
    c = ht - ht.mean(dim=1, keepdim=True) if layer else ht
    yt = c * torch.rsqrt((c * c).mean(dim=1, keepdim=True) + 1e-3) * wt + bt
    ((yt * torch.tensor(dy)).sum() + (ht * torch.tensor(skip)).sum()).backward()
    assert np.abs(y - yt.detach().numpy()).max() < 1e-13
    for got, want in ((dx, xt), (dw, wt), (db, bt)):
        assert np.abs(got - want.grad.numpy()).max() < 1e-13
    # a row's gradient is orthogonal to a constant (layer) and, up to eps, to the row itself
    plain, _, _ = o64.norm_grad(dy, h, w, mu, r, layer)
    if layer:
        assert np.abs(plain.sum(axis=1)).max() < 1e-13
