"""Linear layer and block norms where element offsets pass 2^31: the last rows against fp64, the rows before them finite and written.
Tolerances as in test_gpu_linear.py and test_gpu_block_norm.py, taken as norms: bf16 outputs are off by at most half a step, 2^-8, of each
value (twice that where a bf16 gradient before the activation entered the sum)."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def _near(got, want, steps):
    return ((got.double() - want).norm() / want.norm()).item() <= steps * 2.0 ** -8


@pytest.mark.parametrize("N", [32768, 32771])
def test_linear(N):
    b = gc.binding()
    T, D = 66000, 64
    x = torch.randn(T, D, device=DEV).to(BF)
    W = (torch.randn(N, D, device=DEV) / 8).to(BF)
    y, pre = b.rlf_linear_fwd(x, W, act=b.ACT_SILU, want_pre=True)
    assert y.numel() > 2 ** 31
    tail = slice(T - 40, T)
    z = x[tail].double() @ W.double().t()
    assert _near(y[tail], torch.nn.functional.silu(z), 1) and _near(pre[tail], z, 1)
    assert (y[-3000:].abs().sum(dim=1) > 0).all()
    # gradients of the last rows alone: what the others' zeros add is nothing
    dy = torch.zeros_like(y)
    dy[tail] = torch.randn(40, N, device=DEV).to(BF)
    gx, gw, _ = b.rlf_linear_bwd(dy, x, W, pre=pre, act=b.ACT_SILU)
    s = torch.sigmoid(pre[tail].double())
    gz = dy[tail].double() * s * (1 + pre[tail].double() * (1 - s))
    assert _near(gx[tail], gz @ W.double(), 2) and _near(gw, gz.t() @ x[tail].double(), 2)
    assert not gx[:T - 40].any()


@pytest.mark.parametrize("D", [4096, 4099])
def test_block_norm(D):
    b = gc.binding()
    T = 2 ** 31 // D + 700
    x = torch.randn(T, D, device=DEV, dtype=BF)
    res = torch.randn(T, D, device=DEV, dtype=BF)
    w = (1 + 0.1 * torch.randn(D, device=DEV)).to(BF)
    h, y, stats = b.rlf_block_norm_fwd(x, res, post_weight=w, pre_weight=w)
    rms = lambda v: v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + 1e-6) * w.double()
    for at in (slice(0, 20), slice(T - 20, T)):
        h64 = res[at].double() + rms(x[at].double())
        assert _near(h[at], h64, 1) and _near(y[at], rms(h64), 1)
    del y
    g = b.rlf_block_norm_bwd(h, None, x, h, stats, post_weight=w, pre_weight=w, want_grad_residual=False)
    at = slice(T - 20, T)
    u = h[at].double() * stats[3, at].double()[:, None]
    q = h[at].double() * w.double()
    gh = (q - u * (q * u).mean(dim=1, keepdim=True)) * stats[3, at].double()[:, None]
    v = x[at].double() * stats[1, at].double()[:, None]
    q = gh * w.double()
    want = (q - v * (q * v).mean(dim=1, keepdim=True)) * stats[1, at].double()[:, None]
    assert _near(g["grad_x"][at], want, 1)
    assert g["grad_pre_weight"].isfinite().all() and g["grad_post_weight"].isfinite().all()
