"""rlf_fused_lmhead_cross_entropy on heads with NaN and infinite rows."""
import pytest
import torch

import gpu_common as gc
from test_gpu_fused_cross_entropy import _inputs, check, form, run          # noqa: F401  (form: a fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("V,first,last", [(1032, 1024, 1032), (1032, 256, 512), (1032, 0, 256), (2056, 2048, 2056), (264, 256, 264),
                                          (20008, 19968, 20008)])
def test_nan_rows_that_fill_a_column_tile(form, T, V, first, last):
    """Uninitialised padding rows of the head: a column tile (or a whole split of the vocabulary) holds nothing but NaN.
    Every row of logits has a NaN, so every row is taken out, whichever gradients are asked for."""
    b = gc.binding()
    H, W, ids, mask = _inputs(T, 64, V, 21)
    W[first:last] = float("nan")
    ids.clamp_(max=first - 1) if first else ids.clamp_(min=last)
    for eps in (0.0, 0.1):
        for want_h, want_w, dt in ((True, True, BF), (True, True, F32), (True, False, F32), (False, False, F32)):
            lp, lse, loss, gh, gw = run(H, W, ids, mask, eps, status=b.DEV_NONFINITE, want_grad_hidden=want_h,
                                        want_grad_W=want_w, grad_W_dtype=dt)
            assert torch.isnan(lp).all() and torch.isnan(lse).all() and not loss.any()
            assert gh is None or not gh.any()
            assert gw is None or not gw.any()


@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("V,first,last", [(1032, 0, 64), (1032, 0, 256), (1032, 256, 512), (1032, 1024, 1032), (20008, 19968, 20008)])
def test_masked_columns_without_gradients(T, V, first, last):
    """Columns of -inf (a head whose padding rows hold -inf in a feature that is one) have probability zero, wherever they
    lie; the statistics are those of the other columns."""
    H, W, ids, mask = _inputs(T, 64, V, 22)
    H[:, 3] = 1.0
    ids.clamp_(max=first - 1) if first else ids.clamp_(min=last)
    W[first:last, 3] = float("-inf")
    keep = torch.ones(V, dtype=torch.bool, device=DEV)
    keep[first:last] = False
    at = torch.cumsum(keep, 0).int() - 1
    for zc in (0.0, 1e-3):
        out = run(H, W, ids, mask, 0.0, zc, want_grad_hidden=False, want_grad_W=False)
        check(out, H, W[keep], at[ids.long()], mask, 0.0, zc)


@pytest.mark.parametrize("T,D,V", [(1, 64, 20008), (64, 512, 20008), (257, 320, 4360), (700, 256, 8200), (1500, 64, 1032)])
def test_exactly_the_workspace_asked_for(form, T, D, V):
    """Nothing is written beside the bytes asked for, and the pieces of grad_hidden fit them for any number of live rows."""
    b = gc.binding()
    H, W, ids, mask = _inputs(T, D, V, 23)
    n = b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY, T, V, D, b.RLF_F32)
    buf = torch.full((n + 4096,), 171, dtype=torch.uint8, device=DEV)
    for live in (mask, torch.ones_like(mask), (torch.arange(T, device=DEV) < max(1, T // 9)).to(torch.uint8)):
        check(run(H, W, ids, live, 0.1, 1e-4, workspace=buf[:n]), H, W, ids, live, 0.1, 1e-4)
        assert (buf[n:] == 171).all()


@pytest.mark.parametrize("T,D,V", [(1, 64, 8), (64, 512, 20008), (700, 256, 8200), (19100, 64, 264)])
def test_exactly_the_workspace_of_a_call_without_gradients(form, T, D, V):
    b = gc.binding()
    H, W, ids, mask = _inputs(T, D, V, 24)
    n = b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY_FWD, T, V, D, b.RLF_F32)
    buf = torch.full((n + 4096,), 171, dtype=torch.uint8, device=DEV)
    for live in (mask, torch.ones_like(mask)):
        for eps in (0.0, 0.1):
            out = run(H, W, ids, live, eps, 1e-4, want_grad_hidden=False, want_grad_W=False, workspace=buf[:n])
            check(out, H, W, ids, live, eps, 1e-4)
            assert (buf[n:] == 171).all()
    with pytest.raises(b.RlfError):                   # too small for a gradient
        run(H, W, ids, mask, want_grad_W=False, workspace=buf[:n])


@pytest.mark.parametrize("T,D,V", [(512, 2560, 4104), (300, 64, 1032), (700, 1024, 20008), (64, 4096, 8008)])
def test_tokens_that_the_model_is_sure_of(form, T, D, V):
    """Targets of probability 0.5 to 1 - 1e-13.  dz bounds a logit's error as in check() (tensor-core sums); the log-prob's
    derivative by a logit is [v = y] - p_v, so that errors of the logits move it by at most 2 (1 - p_y) dz; so do relative
    errors of the sum over the other columns against the target's exponential, u = 2^-24: an exponent's rounding u |z - rho| with
    rho = z_y + 32, the target's 32 u, 340 additions, 2^-21 for the exponentials and the logarithm.  It is never above zero.
    A gradient entry p_v (or p_y - 1) carries these twice (its own logit and the row's sum) besides its rounding to bf16 (two
    where the scratch holds dZ itself: the exponential's and the entry's)."""
    b = gc.binding()
    U, HB = 2.0 ** -24, 2.0 ** -8
    g = torch.Generator(device=DEV)
    g.manual_seed(D + T)
    W = (torch.randn(V, D, generator=g, device=DEV) * 2.0 / D ** 0.5).to(BF)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    w = W[ids.long()].float()
    lift = torch.linspace(8, 42, T, device=DEV)[:, None]
    H = (torch.randn(T, D, generator=g, device=DEV) + lift * w / (w * w).sum(1, keepdim=True)).to(BF)
    z = H.double() @ W.double().t()
    y = ids.long()[:, None]
    acc = lambda K: (K / 8 + 16) * 2.0 ** -23
    dz = acc(D) * (H.double().abs() @ W.double().abs().t()).amax(dim=1)
    # 1 - p_y without cancellation
    zy = z.gather(1, y)
    others = torch.exp(z - zy).scatter_(1, y, 0.0).sum(dim=1)
    lp, q = -torch.log1p(others), others / (1 + others)
    p = torch.exp(z - zy) / (1 + others)[:, None]
    rel0 = U * (z.abs().amax(dim=1) + zy[:, 0].abs() + 64 + 340) + 2.0 ** -21
    stored = (2.02 if form == "universal" else 1.01) * HB
    for grad in (True, False):
        logp, lse, loss, gh, gw = run(H, W, ids, None, want_grad_hidden=grad, want_grad_W=grad)
        assert (logp <= 0).all()
        # d log p = q (relative change of the odds)
        rel = torch.expm1(2 * dz) + rel0
        err = (logp.double() - lp).abs()
        assert (err <= q * rel * 1.01 + 3 * U * lp.abs()).all(), (err / (q * rel + 3 * U * lp.abs())).max().item()
        assert ((lse.double() - torch.logsumexp(z, 1)).abs() <= dz + rel0 + 4 * U * z.abs().amax(dim=1)).all()
        if not grad:
            continue
        want = p.clone()
        want.scatter_(1, y, -q[:, None])
        e = p * (2 * rel + stored)[:, None]
        e.scatter_(1, y, (q * (rel + 1.01 * HB))[:, None])
        e = (e + 2.0 ** -126 * 8e13) / T              # (entries that the scratch's range drops)
        want /= T
        mag = want.abs() + e
        got = gh.double()
        ref = want @ W.double()
        bound = e @ W.double().abs() + acc(V) * (mag @ W.double().abs()) + 1.01 * HB * ref.abs()
        over = (got - ref).abs() / bound
        assert (over <= 1).all(), (over.max().item(), torch.nonzero(over > 1)[0].tolist())
