"""GPU parity of rlf_norm_fwd / rlf_norm_bwd against the fp64 definitions in oracle/operators64.py.

Tolerances are error bounds, element by element, with u = 2^-24 (half a step of fp32):
  * a sum over a row is taken by threads that add at most 53 (fast form: 32 elements, 5 shuffles, 16 warps)
    or D / 256 + 13 (general form) terms one after the other: |error| <= CHAIN u sum |terms|, CHAIN = 64
    covers both up to D = 13000; widths beyond that use D / 256 + 14.
  * mean: CHAIN u mean|h|;  r: half the relative error of its mean square, (CHAIN / 2 + 4) u, the 4 for
    rsqrtf (2 ulp) and the division by D.
  * every further operation: u relative.
  * the one rounding to the output's type: half a step, eps / 2 of the value (bf16 2^-8, fp32 2^-24).
"""
import numpy as np
import pytest
import torch

from oracle import operators64 as o64
import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _half(dt):
    return 2.0 ** -8 if dt == BF else U


def _chain(D):
    return 64 if D <= 13000 else D // 256 + 14


def _draw(T, D, dt, w_dt, seed, pad=0, residual=False, bias=False, scale=1.0, offset=0.3):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x = (scale * r(T, D + pad) + offset).to(dt)[:, :D]
    res = (0.7 * r(T, D + pad)).to(dt)[:, :D] if residual else None
    return x, res, (1 + 0.3 * r(D)).to(w_dt), (0.2 * r(D)).to(w_dt) if bias else None


def check_fwd(out, x, res, w, b, layer, eps):
    y, s, mean, rstd = out
    y64, h64, mu64, r64 = o64.norm(_f64(x), _f64(w), _f64(b), _f64(res), layer, eps)
    D, dt = x.shape[1], x.dtype
    C = _chain(D)
    absh = np.abs(h64).mean(axis=1)
    dmu = (C * U * absh) if layer else np.zeros_like(mu64)
    # dmu shifts the mean square by dmu^2 only (the linear term cancels); the rounding of h by u |h| enters twice
    drel = (C / 2 + 4) * U + U * np.abs(h64).max(axis=1) * r64 + 0.5 * (dmu * r64) ** 2
    assert (np.abs(_f64(rstd) - r64) <= 2 * drel * r64).all()
    if layer:
        assert (np.abs(_f64(mean) - mu64) <= dmu + U * np.abs(mu64)).all()
    xh, wn = np.abs((h64 - mu64[:, None]) * r64[:, None]), np.abs(_f64(w))[None, :]
    bound = (_half(dt) * np.abs(y64) + wn * r64[:, None] * (dmu[:, None] + 2 * U * np.abs(h64))
             + wn * xh * (2 * drel[:, None] + 4 * U) + U * np.abs(y64))
    err = np.abs(_f64(y) - y64)
    assert (err <= 1.01 * bound).all(), (err / bound).max()
    if s is not None:
        assert (np.abs(_f64(s) - h64) <= 1.01 * _half(dt) * np.abs(h64) + U * np.abs(h64)).all()


def check_bwd(out, dy, x, w, mean, rstd, layer, skip, rows_chain=700):
    gx, gw, gb = out
    dx64, dw64, db64 = o64.norm_grad(_f64(dy), _f64(x), _f64(w), _f64(mean), _f64(rstd), layer, _f64(skip))
    D, dt = x.shape[1], x.dtype
    C = _chain(D)
    r = _f64(rstd)[:, None]
    mu = _f64(mean)[:, None] if layer else 0.0
    xh = np.abs((_f64(x) - mu) * r)
    g = np.abs(_f64(dy) * _f64(w))
    if gx is not None:
        a = (g * xh).mean(axis=1, keepdims=True)
        b = g.mean(axis=1, keepdims=True) if layer else 0.0
        bound = r * ((C + 8) * U * (b + xh * a) + 8 * U * (g + xh * a + b)) + (_half(dt) + 2 * U) * np.abs(dx64)
        if skip is not None:
            bound = bound + U * np.abs(_f64(skip))
        err = np.abs(_f64(gx) - dx64)
        assert (err <= 1.01 * bound + 1e-45).all(), (err / (bound + 1e-45)).max()
    n = min(rows_chain, x.shape[0] + 160)
    if gw is not None:
        bound = (n + 4) * U * (np.abs(_f64(dy)) * xh).sum(axis=0)
        assert (np.abs(_f64(gw) - dw64) <= bound + 1e-45).all()
    if gb is not None:
        assert (np.abs(_f64(gb) - db64) <= (n + 4) * U * np.abs(_f64(dy)).sum(axis=0) + 1e-45).all()


SIZES = [(1, 1), (1, 64), (3, 7), (5, 1021), (2, 31), (17, 2560), (64, 4096), (9, 8192), (2, 16384), (3, 20001),
         (300, 512), (4097, 128), (33, 2604), (1030, 1022), (700, 5120)]


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("dt,w_dt", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_forward_and_backward(T, D, dt, w_dt, layer):
    b = gc.binding()
    kind = b.NORM_LAYER if layer else b.NORM_RMS
    for k, (pad, residual, bias) in enumerate([(0, False, layer), (8, True, False), (3, True, True)]):
        x, res, w, bias_t = _draw(T, D, dt, w_dt, 10 * T + D + k, pad, residual, bias)
        out = b.rlf_norm_fwd(x, w, bias=bias_t, residual=res, kind=kind, eps=1e-5)
        check_fwd(out, x, res, w, bias_t, layer, 1e-5)
        h = out[1] if residual else x
        dy, skip, _, _ = _draw(T, D, dt, w_dt, 99 + D + k, pad, residual, scale=1e-2, offset=0.0)
        skip = None if skip is None else skip.contiguous()
        got = b.rlf_norm_bwd(dy, h, w, out[2], out[3], kind=kind, grad_skip=skip, want_grad_bias=bias)
        check_bwd(got, dy, h, w, out[2], out[3], layer, skip)
        again = b.rlf_norm_bwd(dy, h, w, out[2], out[3], kind=kind, grad_skip=skip, want_grad_bias=bias)
        for p, q in zip(got, again):
            assert (p is None and q is None) or torch.equal(p, q)


def test_gradient_against_differences():
    """The forward's own differences: sum(dy y(x + h d)) over +-h against the backward's directional derivative."""
    b = gc.binding()
    T, D = 6, 96
    for layer in (False, True):
        kind = b.NORM_LAYER if layer else b.NORM_RMS
        x, _, w, bias = _draw(T, D, F32, F32, 5, bias=True)
        dy, d, _, _ = _draw(T, D, F32, F32, 6, residual=True, offset=0.0)
        y, _, mean, rstd = b.rlf_norm_fwd(x, w, bias=bias, kind=kind)
        gx, gw, gb = b.rlf_norm_bwd(dy, x, w, mean, rstd, kind=kind, want_grad_bias=True)
        f = lambda xx, ww, bb: (b.rlf_norm_fwd(xx, ww, bias=bb, kind=kind)[0].double() * dy.double()).sum().item()
        h = 2.0 ** -7
        # truncation h^2 |f'''| / 6 with third derivatives of order one, rounding 1e-6 |f| / h
        for got, fd in (((gx.double() * d.double()).sum().item(), (f(x + h * d, w, bias) - f(x - h * d, w, bias)) / (2 * h)),
                        (gw.double().sum().item(), (f(x, w + h, bias) - f(x, w - h, bias)) / (2 * h)),
                        (gb.double().sum().item(), (f(x, w, bias + h) - f(x, w, bias - h)) / (2 * h))):
            assert abs(got - fd) <= 2e-3 * (dy.double().norm() * d.double().norm()).item() / 10, (got, fd)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D", [2560, 1021, 20001])
def test_outputs_in_place(dt, D):
    b = gc.binding()
    for layer in (False, True):
        kind = b.NORM_LAYER if layer else b.NORM_RMS
        x, res, w, _ = _draw(37, D, dt, BF, 3, residual=True)
        y, s, mean, rstd = b.rlf_norm_fwd(x, w, residual=res, kind=kind)
        x1, res1 = x.clone(), res.clone()
        y1, s1, _, _ = b.rlf_norm_fwd(x1, w, residual=res1, kind=kind, y_out=x1, sum_out=res1)
        assert torch.equal(y1, y) and torch.equal(s1, s) and y1 is x1 and s1 is res1
        x2, res2 = x.clone(), res.clone()
        y2, s2, _, _ = b.rlf_norm_fwd(x2, w, residual=res2, kind=kind, y_out=res2, sum_out=x2)
        assert torch.equal(y2, y) and torch.equal(s2, s)
        dy, skip, _, _ = _draw(37, D, dt, BF, 4, residual=True)
        ref = b.rlf_norm_bwd(dy, s, w, mean, rstd, kind=kind, grad_skip=skip, want_grad_bias=True)
        for which in range(3):
            a = [dy.clone(), s.clone(), skip.clone()]
            got = b.rlf_norm_bwd(a[0], a[1], w, mean, rstd, kind=kind, grad_skip=a[2], grad_x=a[which], want_grad_bias=True)
            for p, q in zip(got, ref):
                assert torch.equal(p, q)


@pytest.mark.parametrize("D", [256, 1021, 4096, 20001])
def test_a_non_finite_row_stays_in_its_row(D):
    b = gc.binding()
    x, _, w, bias = _draw(12, D, F32, F32, 8, bias=True)
    for layer in (False, True):
        kind = b.NORM_LAYER if layer else b.NORM_RMS
        clean = b.rlf_norm_fwd(x, w, bias=bias, kind=kind)
        bad = x.clone()
        bad[3, D // 2] = float("nan")
        bad[7, 0] = float("inf")
        got = b.rlf_norm_fwd(bad, w, bias=bias, kind=kind)
        keep = torch.ones(12, dtype=torch.bool, device=DEV)
        keep[3] = keep[7] = False
        assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[3][keep], clean[3][keep])
        assert torch.isnan(got[0][3]).all() and not torch.isfinite(got[0][7]).all()
        gx = b.rlf_norm_bwd(x, bad, w, clean[2], clean[3], kind=kind, want_grad_weight=False)[0]
        gc_ = b.rlf_norm_bwd(x, x, w, clean[2], clean[3], kind=kind, want_grad_weight=False)[0]
        assert torch.equal(gx[keep], gc_[keep])


@pytest.mark.parametrize("T,D", [(1, 5), (3, 640), (9, 5), (8, 13), (40, 1021), (301, 2603), (23, 2048), (1200, 77)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_rows_off_their_vectors(T, D, dt, off):
    """All tensors start `off` elements into a 16-byte vector and the strides differ by whole vectors; what lies between
    the rows is NaN and stays as it is."""
    b = gc.binding()
    nan = float("nan")

    def place(src, gap):
        buf = torch.full((off + T * (D + gap) + 16,), nan, dtype=dt, device=DEV)
        v = buf.as_strided((T, D), (D + gap, 1), off)
        v.copy_(src)
        return buf, v

    for layer in (False, True):
        kind = b.NORM_LAYER if layer else b.NORM_RMS
        x0, res0, w, bias = _draw(T, D, dt, BF, 5 * T + D + off, residual=True, bias=True)
        dy0, skip0, _, _ = _draw(T, D, dt, BF, 7 * T + D, residual=True, scale=1e-2, offset=0.0)
        (_, x), (_, res), (by, y), (bs, s) = place(x0, 8), place(res0, 8), place(x0, 0), place(x0, 0)
        out = b.rlf_norm_fwd(x, w, bias=bias, residual=res, kind=kind, y_out=y, sum_out=s)
        check_fwd(out, x0, res0, w, bias, layer, 1e-6)
        (_, dy), (_, sk), (bg, gx) = place(dy0, 16), place(skip0, 0), place(x0, 0)
        got = b.rlf_norm_bwd(dy, s, w, out[2], out[3], kind=kind, grad_skip=sk, grad_x=gx, want_grad_bias=True)
        check_bwd(got, dy0, s, w, out[2], out[3], layer, skip0)
        for buf in (by, bs, bg):
            assert torch.isnan(buf[:off]).all() and torch.isnan(buf[off + T * D:]).all()


def test_constant_zero_and_offset_rows():
    """A constant row (variance zero) gives the bias and no NaN; a large common offset costs the layer form only
    the digits that the fp32 input does not hold."""
    b = gc.binding()
    x = torch.full((3, 1000), 5.0, device=DEV)
    x[1] = 0.0
    w, bias = torch.ones(1000, device=DEV), torch.full((1000,), 0.25, device=DEV)
    y, _, mean, rstd = b.rlf_norm_fwd(x, w, bias=bias, kind=b.NORM_LAYER, eps=1e-6)
    assert (y == 0.25).all() and mean.tolist() == [5.0, 0.0, 5.0]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = 1000.0 + torch.randn(5, 4096, generator=g, device=DEV)
    out = b.rlf_norm_fwd(x, torch.ones(4096, device=DEV), kind=b.NORM_LAYER)
    check_fwd(out, x, None, torch.ones(4096, device=DEV), None, True, 1e-6)


def test_nothing_outside_the_outputs_is_written():
    b = gc.binding()
    for T, D, dt in ((13, 1021, BF), (5, 2560, BF), (7, 999, F32), (2, 20001, BF)):
        x, res, w, bias = _draw(T, D, dt, BF, 2, residual=True, bias=True)
        buf = [torch.full(((T + 2) * D,), 7.0, dtype=dt, device=DEV) for _ in range(3)]
        v = [t[D:D + T * D].view(T, D) for t in buf]
        vec = [torch.full((n + 64,), 7.0, device=DEV) for n in (T, T, D, D)]
        y, s, mean, rstd = b.rlf_norm_fwd(x, w, bias=bias, residual=res, kind=b.NORM_LAYER, y_out=v[0], sum_out=v[1],
                                          mean_out=vec[0][:T], rstd_out=vec[1][:T])
        b.rlf_norm_bwd(y, s, w, mean, rstd, kind=b.NORM_LAYER, grad_x=v[2], grad_weight=vec[2][:D], grad_bias=vec[3][:D])
        for t in buf:
            assert (t[:D] == 7.0).all() and (t[D + T * D:] == 7.0).all()
        for t, n in zip(vec, (T, T, D, D)):
            assert (t[n:] == 7.0).all() and not (t[:n] == 7.0).all()


def test_no_rows_accumulation_and_partial_outputs():
    b = gc.binding()
    D = 640
    x, _, w, _ = _draw(50, D, BF, BF, 9)
    dy, _, _, _ = _draw(50, D, BF, BF, 10)
    y, s, mean, rstd = b.rlf_norm_fwd(x, w)
    assert s is None and mean is None
    _, gw, gb = b.rlf_norm_bwd(dy, x, w, None, rstd, want_grad_bias=True)
    acc_w, acc_b = torch.full((D,), 2.0, device=DEV), torch.full((D,), -1.0, device=DEV)
    gx, _, _ = b.rlf_norm_bwd(dy, x, w, None, rstd, grad_weight=acc_w, grad_bias=acc_b, accumulate=True)
    assert torch.equal(acc_w, 2.0 + gw) and torch.equal(acc_b, gb - 1.0)
    only_x = b.rlf_norm_bwd(dy, x, w, None, rstd, want_grad_weight=False)
    assert torch.equal(only_x[0], gx) and only_x[1] is None and only_x[2] is None
    only_w = b.rlf_norm_bwd(dy, x, w, None, rstd, want_grad_x=False)
    assert only_w[0] is None and torch.equal(only_w[1], gw)
    e = torch.empty((0, D), dtype=BF, device=DEV)
    assert b.rlf_norm_fwd(e, w)[0].shape == (0, D)
    z, zw, zb = b.rlf_norm_bwd(e, e, w, None, torch.empty(0, device=DEV), want_grad_bias=True)
    assert z.shape == (0, D) and not zw.any() and not zb.any()
    b.rlf_norm_bwd(e, e, w, None, torch.empty(0, device=DEV), grad_weight=acc_w, want_grad_bias=False, accumulate=True)
    assert torch.equal(acc_w, 2.0 + gw)


def test_captured_and_replayed_and_on_two_streams():
    b = gc.binding()
    T, D = 500, 2560
    x, res, w, _ = _draw(T, D, BF, BF, 11, residual=True)
    dy, _, _, _ = _draw(T, D, BF, BF, 12)
    eager = b.rlf_norm_fwd(x, w, residual=res)
    eager_b = b.rlf_norm_bwd(dy, eager[1], w, None, eager[3])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            o = b.rlf_norm_fwd(x, w, residual=res)
            b.rlf_norm_bwd(dy, o[1], w, None, o[3])
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = b.rlf_norm_fwd(x, w, residual=res)
        ob = b.rlf_norm_bwd(dy, o[1], w, None, o[3])
    x2, dy2 = x.flip(0).clone(), dy.flip(0).clone()
    keep = (x.clone(), dy.clone())
    x.copy_(x2), dy.copy_(dy2)
    res.copy_(res.flip(0).clone())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o[0], eager[0].flip(0)) and torch.equal(ob[0], eager_b[0].flip(0))
    x.copy_(keep[0]), dy.copy_(keep[1])
    res.copy_(res.flip(0).clone())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o[0], eager[0]) and torch.equal(ob[0], eager_b[0]) and torch.equal(ob[1], eager_b[1])
    # two calls at once, each on a stream and with a workspace of its own
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for st in streams:
        with torch.cuda.stream(st):
            for _ in range(5):
                outs.append(b.rlf_norm_bwd(dy, eager[1], w, None, eager[3]))
    torch.cuda.synchronize()
    for got in outs:
        assert torch.equal(got[0], eager_b[0]) and torch.equal(got[1], eager_b[1])


def test_rows_past_32_bit_offsets():
    """More than 2^31 elements: the last rows of a [T, D] batch sit beyond a 32-bit element offset."""
    b = gc.binding()
    D, T = 4096, (1 << 19) + 77
    x = torch.empty((T, D), dtype=BF, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(4))
    w = torch.ones(D, dtype=BF, device=DEV)
    y, _, _, rstd = b.rlf_norm_fwd(x, w)
    tail = b.rlf_norm_fwd(x[-90:].clone(), w)
    assert torch.equal(y[-90:], tail[0]) and torch.equal(rstd[-90:], tail[3])
    gx, gw, _ = b.rlf_norm_bwd(y, x, w, None, rstd)
    tg = b.rlf_norm_bwd(y[-90:].clone(), x[-90:].clone(), w, None, rstd[-90:].clone())
    assert torch.equal(gx[-90:], tg[0])
    # y xh = xh^2 sums to about T in every column; five standard deviations of a chi-square with T degrees
    assert (gw - T).abs().max().item() < 5 * (2 * T) ** 0.5 + 2.0 ** -8 * T
