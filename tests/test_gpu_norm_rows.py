"""GPU parity of rlf_norm_fwd / rlf_norm_bwd on rows in unusual places, with the bounds of tests/test_gpu_norm.py."""
import pytest
import torch

import gpu_common as gc
from test_gpu_norm import check_bwd, check_fwd

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


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


# The bounds of tests/test_gpu_norm.py, evaluated for all rows in 64 bits on the GPU.
def _half(dt):
    return 2.0 ** -8 if dt == BF else U


def check_fwd_rows(out, x, res, w, bias, layer, eps, C=64):
    y, s, mean, rstd = out
    dt = x.dtype
    for a in range(0, x.shape[0], 8192):
        k = slice(a, a + 8192)
        h = x[k].double() + (0.0 if res is None else res[k].double())
        mu = h.mean(dim=1, keepdim=True) if layer else torch.zeros(h.shape[0], 1, dtype=torch.float64, device=DEV)
        c = h - mu
        r = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + eps)
        want = c * r * w.double() + (0.0 if bias is None else bias.double())
        dmu = C * U * h.abs().mean(dim=1, keepdim=True) if layer else 0.0 * mu
        drel = (C / 2 + 4) * U + U * h.abs().max(dim=1, keepdim=True).values * r + 0.5 * (dmu * r) ** 2
        assert ((rstd[k].double()[:, None] - r).abs() <= 2 * drel * r).all()
        if layer:
            assert ((mean[k].double()[:, None] - mu).abs() <= dmu + U * mu.abs()).all()
        wn = w.double().abs()
        bound = (_half(dt) * want.abs() + wn * r * (dmu + 2 * U * h.abs()) + wn * (c * r).abs() * (2 * drel + 4 * U) + U * want.abs())
        bad = (y[k].double() - want).abs() > 1.01 * bound
        assert not bad.any(), (a + torch.nonzero(bad)[0, 0].item(), int(bad.sum()))
        if s is not None:
            assert ((s[k].double() - h).abs() <= 1.01 * _half(dt) * h.abs() + U * h.abs()).all()


def check_bwd_rows(out, dy, x, w, mean, rstd, layer, skip, C=64, rows_chain=700):
    gx, gw, gb = out
    T, D = x.shape
    dt = x.dtype
    f64 = lambda *n: torch.zeros(*n, dtype=torch.float64, device=DEV)
    dw, db, dw_abs, db_abs = f64(D), f64(D), f64(D), f64(D)
    for a in range(0, T, 8192):
        k = slice(a, a + 8192)
        r = rstd[k].double()[:, None]
        xh = (x[k].double() - (mean[k].double()[:, None] if layer else 0.0)) * r
        d = dy[k].double()
        g = d * w.double()
        want = g - xh * (g * xh).mean(dim=1, keepdim=True)
        if layer:
            want = want - g.mean(dim=1, keepdim=True)
        want = want * r + (0.0 if skip is None else skip[k].double())
        m = (g * xh).abs().mean(dim=1, keepdim=True)
        n = g.abs().mean(dim=1, keepdim=True) if layer else 0.0 * m
        bound = r * ((C + 8) * U * (n + xh.abs() * m) + 8 * U * (g.abs() + xh.abs() * m + n)) + (_half(dt) + 2 * U) * want.abs()
        if skip is not None:
            bound = bound + U * skip[k].double().abs()
        bad = (gx[k].double() - want).abs() > 1.01 * bound + 1e-45
        assert not bad.any(), (a + torch.nonzero(bad)[0, 0].item(), int(bad.sum()))
        dw += (d * xh).sum(dim=0)
        db += d.sum(dim=0)
        dw_abs += (d * xh).abs().sum(dim=0)
        db_abs += d.abs().sum(dim=0)
    n = min(rows_chain, T + 160) + 4
    assert ((gw.double() - dw).abs() <= n * U * dw_abs + 1e-45).all()
    if gb is not None:
        assert ((gb.double() - db).abs() <= n * U * db_abs + 1e-45).all()


# every form and cut of the rows, several batches per CTA: aligned, on no boundary, staged
@pytest.mark.parametrize("dt,w_dt", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("T,D", [(150001, 64), (100003, 328), (60001, 768), (40003, 1021), (40001, 1022), (40002, 1024), (24001, 2048),
                                 (20001, 2560), (16001, 2603), (9001, 5120), (7001, 8192)])
@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_many_rows_per_cta(T, D, dt, w_dt, layer):
    b = gc.binding()
    kind = b.NORM_LAYER if layer else b.NORM_RMS
    vec = 16 // (2 if dt == BF else 4)
    for seed, (pad, residual, bias) in enumerate([(0, False, layer), (vec, True, layer), (3, True, True), (3, False, False)]):
        g = torch.Generator(device=DEV)
        g.manual_seed(D + seed)
        r = lambda *n: torch.randn(*n, generator=g, device=DEV)
        x = (r(T, D + pad) + 0.3).to(dt)[:, :D]
        res = (0.7 * r(T, D + pad)).to(dt)[:, :D] if residual else None
        w, bias_t = (1 + 0.3 * r(D)).to(w_dt), (0.2 * r(D)).to(w_dt) if bias else None
        out = b.rlf_norm_fwd(x, w, bias=bias_t, residual=res, kind=kind, eps=1e-5)
        check_fwd_rows(out, x, res, w, bias_t, layer, 1e-5)
        h = out[1] if residual else x
        dy = (1e-2 * r(T, D + pad)).to(dt)[:, :D]
        skip = (1e-2 * r(T, D)).to(dt) if residual else None
        got = b.rlf_norm_bwd(dy, h, w, out[2], out[3], kind=kind, grad_skip=skip, want_grad_bias=bias)
        check_bwd_rows(got, dy, h, w, out[2], out[3], layer, skip)
        if residual:
            # in place: the gradient over the residual stream's, the sum over its input
            again = b.rlf_norm_bwd(dy, h, w, out[2], out[3], kind=kind, grad_skip=skip, grad_x=skip, want_grad_bias=bias)
            assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
        elif pad == 0:
            y = b.rlf_norm_fwd(x, w, bias=bias_t, kind=kind, eps=1e-5, y_out=x)[0]
            assert torch.equal(y, out[0])
