"""NaN and infinities in some rows of the linear layer's backward and of long batches through the block norms (several rows to a CTA at a
time): every other row's result is bit for bit what it is without them."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("N", [1, 2, 71, 264])
@pytest.mark.parametrize("T", [6, 300, 3000])
def test_linear_backward(T, N, gated):
    b = gc.binding()
    g = torch.Generator(device=DEV)
    g.manual_seed(T + N)
    r = lambda *s, k=1.0: (torch.randn(*s, generator=g, device=DEV) * k).to(BF)
    rows, D = 2 * N if gated else N, 128
    x, W, dy = r(T, D), r(rows, D, k=0.1), r(T, N)
    _, pre = b.rlf_linear_fwd(x, W, act=b.ACT_SILU, gated=gated, want_pre=True)
    args = dict(act=b.ACT_SILU, gated=gated, want_grad_bias=True)
    clean = b.rlf_linear_bwd(dy, x, W, pre=pre, **args)
    dy[2, 0], dy[T - 1, N - 1], pre[4, rows - 1] = NAN, INF, NAN
    got = b.rlf_linear_bwd(dy, x, W, pre=pre, **args)
    rest = [t for t in range(T) if t not in (2, 4, T - 1)]
    assert torch.equal(got[0][rest], clean[0][rest])
    assert got[0][2].isnan().all() and got[0][4].isnan().all()
    # a row of grad_W belongs to a column of grad_y (gated: to a gate and an up row), and only those that met a NaN have one
    met = torch.zeros(rows, dtype=torch.bool, device=DEV)
    for n in (0, (rows - 1) % N, N - 1):
        met[n::N] = True
    assert torch.equal(got[1][~met], clean[1][~met]) and torch.equal(got[2][~met], clean[2][~met])
    assert got[1][0].isnan().all() and got[2][0].isnan()


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "rms"), ("rms", None), (None, "layer")])
@pytest.mark.parametrize("T,D,pad", [(5000, 512, 0), (5000, 509, 0), (5000, 512, 3), (3001, 1021, 1), (700, 8192, 0)])
def test_block_norm(T, D, pad, post, pre, dt):
    b = gc.binding()
    g = torch.Generator(device=DEV)
    g.manual_seed(T + D)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    kinds = {None: b.NORM_NONE, "rms": b.NORM_RMS, "layer": b.NORM_LAYER}
    w1, w2, gate = 1 + 0.1 * r(D), 1 + 0.1 * r(D), r(T)
    x, res = r(T, D + pad).to(dt)[:, :D], r(T, D).to(dt)
    dy, dh = r(T, D).to(dt), r(T, D).to(dt)
    form = dict(post_weight=w1 if post else None, pre_weight=w2 if pre else None, post_kind=kinds[post], pre_kind=kinds[pre], gate=gate,
                gate_form=b.GATE_ROW)

    def both():
        h, y, stats = b.rlf_block_norm_fwd(x, res, **form)
        k = b.rlf_block_norm_bwd(dy if pre else None, dh, x, h, stats, **form)
        return [h, y, stats.t(), k["grad_x"], k["grad_residual"], k["grad_gate"]]

    clean = both()
    bad = [0, 7, 8, 1184, 2000, T - 2] if T > 2000 else [0, 7, 8, T - 2]
    for i, t in enumerate(bad):
        x[t, (0, D - 1, D // 2)[i % 3]] = (NAN, INF)[i % 2]
    for i, t in enumerate((11, 12, T - 1)):
        res[t, (D - 1, 0, D // 2)[i]] = (INF, NAN, -INF)[i]
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[bad + [11, 12, T - 1]] = False
    for p, q in zip(both(), clean):
        assert p is None and q is None or torch.equal(p[rest], q[rest])
