"""Sums over tokens and inputs of the linear layer and the block norms on small whole numbers: every partial sum is a whole number below
2^24, which fp32 holds whatever the order, so that the results have to be equal, and a token that is left out or counted twice
shows at any length.  (bf16 results are the exact ones rounded once.)"""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _whole(g, most, *shape):
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV)


def _gen(*seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(p * s for p, s in zip((1, 31, 1009), seed)))
    return g


def _both(T, D, N, gated=False, dy_dt=BF, gw_dt=F32, accumulate=False):
    b = gc.binding()
    g = _gen(T, D, N)
    rows = 2 * N if gated else N
    x, W, dy, pre = _whole(g, 2, T, D), _whole(g, 2, rows, D), _whole(g, 2, T, N), _whole(g, 2, T, rows)
    gz = torch.cat([dy * pre[:, N:], dy * pre[:, :N]], dim=1) if gated else dy
    d = lambda t: t.double()
    xb, Wb = x.to(BF), W.to(BF)
    y, z = b.rlf_linear_fwd(xb, Wb, gated=gated, out_dtype=F32, want_pre=True)
    want_z = d(x) @ d(W).t()
    assert torch.equal(z, want_z.float().to(BF))
    if not gated:                                               # (the product of two such sums may pass 2^24)
        assert torch.equal(y, want_z.float())
    out = dict(grad_W_dtype=gw_dt, want_grad_bias=True)
    before_w = before_b = 0.0
    if accumulate:
        before_w, before_b = _whole(g, 9, rows, D).float(), _whole(g, 9, rows).float()
        out = dict(grad_W=before_w.clone(), grad_bias=before_b.clone(), accumulate=True)
    gx, gw, gb = b.rlf_linear_bwd(dy.to(dy_dt), xb, Wb, pre=pre.to(BF) if gated else None, gated=gated, **out)
    assert torch.equal(gx, (d(gz) @ d(W)).float().to(BF))
    assert torch.equal(gw, (d(gz).t() @ d(x) + before_w).float().to(gw.dtype))
    assert torch.equal(gb, (d(gz).sum(dim=0) + before_b).float())


@pytest.mark.parametrize("N", [1, 2, 3, 4])
@pytest.mark.parametrize("T,D", [(20011, 72), (8191, 8192), (600, 262144), (32768, 2560), (40000, 8), (9000, 4104), (65, 16)])
def test_few_outputs(T, D, N):
    """Slices of more than 64 tokens, which are taken in several turns, the last of them short; columns without a thread and threads
    without a column."""
    _both(T, D, N, dy_dt=(BF, F32)[N % 2], gw_dt=(F32, BF)[T % 2])
    _both(T, D, N, accumulate=True)


@pytest.mark.parametrize("T,D,N", [(20011, 72, 5), (5000, 136, 1031), (8191, 512, 264), (33, 2560, 130), (100000, 64, 72), (300, 10240, 40)])
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_products(T, D, N, gated):
    _both(T, D, N, gated, dy_dt=(BF, F32)[T % 2])
    _both(T, D, N, gated, accumulate=True)


@pytest.mark.parametrize("form,tile,split", [(1, 256, 0), (1, 128, 0), (3, 256, 0), (2, 64, 8), (2, 256, 3)])
def test_products_in_every_form(form, tile, split):
    b = gc.binding()
    b.tune_linear(form, tile, split)
    try:
        for gated in (False, True):
            _both(2011, 328, 137, gated)
            _both(2011, 328, 136, gated, accumulate=True)
    finally:
        b.tune_linear(0, 0, 0)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("T,D", [(1, 64), (20011, 72), (60000, 256), (5768, 128), (9001, 1021), (4099, 4096), (3000, 7104), (2111, 9000), (50000, 5)])
def test_block_norm_sums(T, D, dt):
    """With statistics of 0 and 1 and one norm absent the weights' and biases' gradients are plain sums of products."""
    b = gc.binding()
    g = _gen(T, D)
    x, dh, dy = _whole(g, 2, T, D), _whole(g, 2, T, D), _whole(g, 2, T, D)
    c = lambda t: t.to(dt)
    stats = torch.zeros(4, T, device=DEV)
    stats[1] = stats[3] = 1.0
    one = torch.ones(D, device=DEV)
    sums = lambda a, w: (a.double() * w.double()).sum(dim=0).float()
    for bias in (False, True):
        for acc in (False, True):
            buf = lambda: _whole(g, 9, D).float()
            kw = dict(want_grad_bias=bias, accumulate=acc, post_kind=b.NORM_RMS, pre_kind=b.NORM_NONE)
            w0, b0, g0 = buf(), buf(), buf()
            if acc:
                kw.update(grad_post_weight=w0.clone(), grad_gate=g0.clone())
                if bias:
                    kw.update(grad_post_bias=b0.clone())
            k = b.rlf_block_norm_bwd(None, c(dh), c(x), None, stats, post_weight=one, gate=one, gate_form=b.GATE_COLUMN, **kw)
            assert torch.equal(k["grad_post_weight"], sums(dh, x) + (w0 if acc else 0))
            assert torch.equal(k["grad_gate"], sums(dh, x) + (g0 if acc else 0))
            if bias:
                assert torch.equal(k["grad_post_bias"], dh.double().sum(dim=0).float() + (b0 if acc else 0))
            kw = dict(want_grad_bias=bias, accumulate=acc, post_kind=b.NORM_NONE, pre_kind=b.NORM_LAYER)
            if acc:
                kw.update(grad_pre_weight=w0.clone())
                if bias:
                    kw.update(grad_pre_bias=b0.clone())
            k = b.rlf_block_norm_bwd(c(dy), None, c(dh), c(x), stats, pre_weight=one, **kw)
            assert torch.equal(k["grad_pre_weight"], sums(dy, x) + (w0 if acc else 0))
            if bias:
                assert torch.equal(k["grad_pre_bias"], dy.double().sum(dim=0).float() + (b0 if acc else 0))
