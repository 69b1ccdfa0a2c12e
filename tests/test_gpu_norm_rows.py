"""GPU parity of rlf_norm_fwd / rlf_norm_bwd on rows in unusual places, with the bounds of tests/test_gpu_norm.py."""
import pytest
import torch

import gpu_common as gc
from test_gpu_norm import check_bwd, check_fwd

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _place(t, stride, offset, before):
    """t [T, D] with rows `stride` elements apart, `offset` elements into a buffer that holds `before` up to there."""
    T, D = t.shape
    buf = torch.full((offset + (T - 1) * stride + D + 8,), before, dtype=t.dtype, device=DEV)
    v = buf.as_strided((T, D), (stride, 1), offset)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_rows_shorter_than_a_vector_on_any_base(dt, layer):
    """Several rows share the 16-byte vector that the tensors start in; what lies before is not part of a row."""
    b = gc.binding()
    kind = b.NORM_LAYER if layer else b.NORM_RMS
    vec = 16 // (2 if dt == BF else 4)
    nan = float("nan")
    for D in (1, 2, 3, 7):
        for offset in range(vec):
            for more in (0, 1, vec):                      # dense rows, rows that go staged, rows alike in their vectors
                g = torch.Generator(device=DEV)
                g.manual_seed(100 * D + 10 * offset + more)
                r = lambda: torch.randn(41, D, generator=g, device=DEV).to(dt)
                x, res = (_place(r() + 0.5, D + more, offset, nan) for _ in range(2))
                w, bias = r()[0].contiguous(), r()[0].contiguous()
                y = _place(r(), D, offset, nan)
                s = _place(r(), D, offset, nan)
                out = b.rlf_norm_fwd(x, w, bias=bias, residual=res, kind=kind, eps=1e-2, y_out=y, sum_out=s)
                check_fwd(out, x, res, w, bias, layer, 1e-2)
                dy = _place(r(), D + more, offset, nan)
                skip = _place(r(), D, offset, nan)
                gx = _place(r(), D, offset, nan)
                got = b.rlf_norm_bwd(dy, s, w, out[2], out[3], kind=kind, grad_skip=skip, want_grad_bias=True, grad_x=gx)
                check_bwd(got, dy, s, w, out[2], out[3], layer, skip)
