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
