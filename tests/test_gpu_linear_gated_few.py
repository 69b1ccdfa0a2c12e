"""Gated linear layers of one to four outputs, forward and backward (plain ones of as many take a path of their own, these the
tensor cores'): against the fp64 definitions with the bounds of test_gpu_linear.py, in a workspace of exactly the stated size
between strips that have to stay as they are."""
import pytest
import torch

from oracle import blocks64 as b64
import gpu_common as gc
from test_gpu_linear import ACTS, BF, DEV, F32, _draw, _f64, both_ways, check_bwd, check_fwd

pytestmark = pytest.mark.gpu
STRIP = 1 << 16


def _exact_workspace(b, T, rows, D):
    n = b.workspace_bytes(b.FN_LINEAR_BWD, T, rows, D, b.RLF_BF16)
    whole = torch.full((n + 2 * STRIP,), 0xA5, dtype=torch.uint8, device=DEV)
    return whole, whole[STRIP:STRIP + n]


def _strips_untouched(whole):
    return bool((whole[:STRIP] == 0xA5).all() and (whole[-STRIP:] == 0xA5).all())


@pytest.mark.parametrize("N", [1, 2, 3, 4])
@pytest.mark.parametrize("T,D", [(1, 8), (33, 64), (300, 8), (5000, 64), (4096, 2560)])
def test_backward_keeps_to_its_workspace(T, D, N):
    b = gc.binding()
    for dt, pad, kind in ((BF, 0, b64.SILU), (F32, 1, b64.GELU_TANH), (BF, 3, b64.NONE)):
        x, W, bias, _ = _draw(T, D, N, gated=True, bias=F32, seed=3)
        _, pre = b.rlf_linear_fwd(x, W, bias=bias, act=kind, gated=True, want_pre=True)
        dy = torch.randn(T, N + pad, device=DEV).to(dt)[:, :N]
        args = dict(pre=pre, act=kind, gated=True)
        for want_bias in (False, True):
            whole, ws = _exact_workspace(b, T, 2 * N, D)
            out = b.rlf_linear_bwd(dy, x, W, want_grad_bias=want_bias, workspace=ws, **args)
            check_bwd(out, dy, x, W, pre, kind, True)
            assert _strips_untouched(whole)
        gw, gb = torch.randn(2 * N, D, device=DEV), torch.randn(2 * N, device=DEV)
        before = _f64(gw), _f64(gb)
        whole, ws = _exact_workspace(b, T, 2 * N, D)
        out = b.rlf_linear_bwd(dy, x, W, grad_W=gw, grad_bias=gb, accumulate=True, workspace=ws, **args)
        check_bwd(out, dy, x, W, pre, kind, True, before)
        assert _strips_untouched(whole)


@pytest.mark.parametrize("N", [1, 2])
def test_more_tokens_than_partial_rows_could_hide(N):
    """T x 16 bytes of gz beside a workspace whose partial rows are far smaller."""
    b = gc.binding()
    T, D = 32768, 64
    x, W, bias, _ = _draw(T, D, N, gated=True, bias=BF, seed=4)
    y, pre = b.rlf_linear_fwd(x, W, bias=bias, act=b64.SILU, gated=True, want_pre=True)
    check_fwd(y, pre, x, W, bias, b64.SILU, True, None)
    dy = torch.randn(T, N, device=DEV).to(BF)
    whole, ws = _exact_workspace(b, T, 2 * N, D)
    out = b.rlf_linear_bwd(dy, x, W, pre=pre, act=b64.SILU, gated=True, want_grad_bias=True, workspace=ws)
    check_bwd(out, dy, x, W, pre, b64.SILU, True)
    assert _strips_untouched(whole)
    again = b.rlf_linear_bwd(dy, x, W, pre=pre, act=b64.SILU, gated=True, want_grad_bias=True)
    assert all(torch.equal(p, q) for p, q in zip(out, again))


@pytest.mark.parametrize("N", [1, 2, 3, 4])
@pytest.mark.parametrize("T,D", [(1, 8), (7, 64), (65, 2560), (333, 4096), (5000, 136), (9000, 24)])
def test_both_ways(T, D, N):
    both_ways(T, D, N, ACTS[N], True, bias=F32, out=F32, grad_w=BF)
    both_ways(T, D, N, ACTS[(N + T) % 5], True, bias=BF, residual=BF, pad=16, seed=2, dy_pad=1, res_pad=1)


@pytest.mark.parametrize("form", [1, 2, 3])
@pytest.mark.parametrize("N", [1, 2, 4])
def test_every_form(form, N):
    """Gate and up rows share one box of the copies of W; every form of the products."""
    b = gc.binding()
    b.tune_linear(form, 0, 0)
    try:
        for T in (3, 70, 600):
            both_ways(T, 72, N, b64.GELU, True, bias=BF, residual=F32, out=F32)
    finally:
        b.tune_linear(0, 0, 0)
