"""Pins of the fp64 definitions in oracle/blocks64.py: fp64 autograd, differences and closed forms."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import blocks64 as b64

TORCH_ACT = {b64.NONE: lambda z: z, b64.RELU: F.relu, b64.SILU: F.silu, b64.GELU: F.gelu,
             b64.GELU_TANH: lambda z: F.gelu(z, approximate="tanh")}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", sorted(TORCH_ACT))
def test_linear_against_autograd(kind, gated):
    rng = np.random.default_rng(5 + kind)
    T, D, N = 5, 7, 4
    rows = 2 * N if gated else N
    x, W, b, r = (rng.normal(size=s) for s in ((T, D), (rows, D), (rows,), (T, N)))
    dy = rng.normal(size=(T, N))
    xt, Wt, bt, rt = (torch.tensor(a, requires_grad=True) for a in (x, W, b, r))
    z = F.linear(xt, Wt, bt)
    y = (TORCH_ACT[kind](z[:, :N]) * z[:, N:] if gated else TORCH_ACT[kind](z)) + rt
    y.backward(torch.tensor(dy))
    got, z64 = b64.linear(x, W, b, kind, gated, r)
    assert np.abs(got - y.detach().numpy()).max() < 1e-13
    gx, gw, gb, _ = b64.linear_grad(dy, x, W, z64, kind, gated)
    for a, t in ((gx, xt), (gw, Wt), (gb, bt)):
        assert np.abs(a - t.grad.numpy()).max() < 1e-12
    assert np.abs(rt.grad.numpy() - dy).max() == 0


def test_activations_far_out():
    far = np.array([-1e4, -200.0, -40.0, 40.0, 1e4])
    for kind in (b64.RELU, b64.SILU, b64.GELU, b64.GELU_TANH):
        assert np.allclose(b64.act(far, kind)[3:], far[3:]) and np.abs(b64.act(far, kind)[:3]).max() < 1e-15
        assert np.allclose(b64.act_grad(far, kind), [0, 0, 0, 1, 1], atol=1e-12)


@pytest.mark.parametrize("form", [None, "column", "row"])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("rms", None), (None, "layer"), ("layer", "rms")])
def test_block_norm_against_autograd(post, pre, form):
    rng = np.random.default_rng(11)
    T, D, alpha, beta, eps = 4, 9, 0.75, 1.5, 1e-3
    x, res, dy, dh = (rng.normal(size=(T, D)) for _ in range(4))
    w1, b1, w2, b2 = (rng.normal(size=D) for _ in range(4))
    gate = None if form is None else rng.normal(size=D if form == "column" else T)
    t = {k: torch.tensor(v, requires_grad=True) for k, v in dict(x=x, res=res, w1=w1, b1=b1, w2=w2, b2=b2).items()}
    gt = None if gate is None else torch.tensor(gate, requires_grad=True)

    def norm(v, kind, w, b):
        if kind is None:
            return v
        c = v - v.mean(dim=1, keepdim=True) if kind == "layer" else v
        return c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + eps) * w + b

    n = norm(t["x"], post, t["w1"], t["b1"])
    g = 1.0 if gt is None else (gt[None, :] if form == "column" else gt[:, None])
    h = alpha * t["res"] + beta * g * n
    y = norm(h, pre, t["w2"], t["b2"])
    total = (h * torch.tensor(dh)).sum() + ((y * torch.tensor(dy)).sum() if pre else 0.0)
    total.backward()
    args = dict(post=post, post_w=w1, post_b=b1, pre=pre, pre_w=w2, gate=gate, form=form, alpha=alpha, beta=beta)
    h64, y64, stats = b64.block_norm(x, res, pre_b=b2, eps=eps, **args)
    assert np.abs(h64 - h.detach().numpy()).max() < 1e-13
    if pre:
        assert np.abs(y64 - y.detach().numpy()).max() < 1e-13
    else:
        assert y64 is None
    r = b64.block_norm_grad(dy if pre else None, dh, x, h64, stats, **args)
    names = dict(x="x", residual="res", post_weight="w1", post_bias="b1", pre_weight="w2", pre_bias="b2")
    for k, v in r.items():
        want = gt.grad if k == "gate" else t[names[k]].grad
        assert np.abs(v - want.numpy()).max() < 1e-12, k
    # the norm's own invariants
    if pre == "layer":
        u = (h64 - stats[2][:, None]) * stats[3][:, None]
        assert np.abs(u.mean(axis=1)).max() < 1e-12
