"""GPU parity of rlf_linear_fwd / rlf_linear_bwd against the fp64 definitions in oracle/blocks64.py.

Tolerances are error bounds, element by element, with u = 2^-24 (half a step of fp32):
  * a product's sum: bf16 x bf16 is exact in fp32; the tensor cores add 16 terms to the running sum at a time and truncate
    (a step of fp32, 2 u, of what is added up; four times that for the alignment of the 16 terms), so after K terms and the
    join of up to 8 parts |error| <= 8 u (K / 16 + 8) sum |terms|.
  * activations: |act'| <= 1.13; their own error relative to the value: sigmoid is e^x to 2 ulp plus the rounding of its argument
    (|x| u, doubled for the tanh form's cubic: 8 |x| u) plus the reciprocal: (16 + 8 |x|) u covers it; Phi 5 ulp = 10 u.
  * every rounding to bf16: 2^-8 of the value; gz is rounded once before it enters a product.
"""
import numpy as np
import pytest
import torch

from oracle import blocks64 as b64
import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
ACTS = [b64.NONE, b64.RELU, b64.SILU, b64.GELU, b64.GELU_TANH]


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _half(dt):
    return 2.0 ** -8 if dt == BF else U


def _draw(T, D, N, gated=False, pad=0, bias=None, residual=None, seed=0, res_pad=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000 * seed + 7 * T + 3 * D + N)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    rows = 2 * N if gated else N
    x = r(T, D + pad).to(BF)[:, :D]
    W = (1.3 / D ** 0.5 * r(rows, D)).to(BF)
    b = None if bias is None else (0.5 * r(rows)).to(bias)
    res = None if residual is None else r(T, N + res_pad).to(residual)[:, :N]
    return x, W, b, res


def _sum_error(K, terms):
    return 8 * U * (K / 16 + 8) * terms


def _act_error(z, kind):
    """own relative error of an activation (and of its derivative's parts) at z"""
    a = np.abs(z)
    if kind in (b64.NONE, b64.RELU):
        return np.zeros_like(z)
    if kind == b64.GELU:
        return np.full_like(z, 16 * U) + 2 * U * z * z
    arg = a if kind == b64.SILU else 1.6 * a * (1 + 0.045 * z * z)
    return (16 + 8 * arg) * U


def check_fwd(y, pre, x, W, bias, kind, gated, residual):
    X, w = _f64(x), _f64(W)
    y64, z64 = b64.linear(X, w, _f64(bias), kind, gated, _f64(residual))
    D, N = X.shape[1], y64.shape[1]
    dz = _sum_error(D, np.abs(X) @ np.abs(w).T) + 2 * U * np.abs(z64)
    if pre is not None:
        assert (np.abs(_f64(pre) - z64) <= 1.01 * (dz + 2.0 ** -8 * np.abs(z64))).all()
    zg = z64[:, :N]
    value = np.abs(b64.act(zg, kind))
    d = 1.13 * dz[:, :N] + _act_error(zg, kind) * value
    if gated:
        d = d * np.abs(z64[:, N:]) + value * dz[:, N:] + d * dz[:, N:]
        value = value * np.abs(z64[:, N:])
    bound = d + 2 * U * (value + np.abs(y64)) + _half(y.dtype) * np.abs(y64) + 1e-30
    err = np.abs(_f64(y) - y64)
    assert (err <= 1.01 * bound).all(), (err / bound).max()


def check_bwd(out, dy, x, W, pre, kind, gated, before=None):
    gx, gw, gb = out
    X, w, z, g = _f64(x), _f64(W), _f64(pre), _f64(dy)
    gx64, gw64, gb64, gz = b64.linear_grad(g, X, w, z, kind, gated)
    T, N = g.shape
    few = not gated and N <= 4
    own = np.zeros_like(gz)
    if kind != b64.NONE or gated:
        zg = z[:, :N]
        # the derivative is a sum of parts up to 1 + |z| large
        slope = (_act_error(zg, kind) + 8 * U) * (1 + np.abs(zg)) * np.abs(g)
        own = np.concatenate([slope * np.abs(z[:, N:]), (_act_error(zg, kind) + 4 * U) * np.abs(g * b64.act(zg, kind))], axis=1) if gated else slope
    exact = few or (kind == b64.NONE and not gated and dy.dtype == BF)
    dgz = own + (0.0 if exact else 2.0 ** -8) * np.abs(gz) + 1e-40
    if gx is not None:
        bound = dgz @ np.abs(w) + _sum_error(gz.shape[1], np.abs(gz) @ np.abs(w)) + 2.0 ** -8 * np.abs(gx64)
        err = np.abs(_f64(gx) - gx64)
        assert (err <= 1.01 * bound + 1e-35).all(), (err / (bound + 1e-35)).max()
    if gw is not None:
        if before is not None:
            gw64 = gw64 + before[0]
        # (few outputs: fp32 sums of at most T terms in turn)
        bound = dgz.T @ np.abs(X) + _sum_error(T, np.abs(gz).T @ np.abs(X)) + (_half(gw.dtype) + 2 * U) * np.abs(gw64)
        if few:
            bound = bound + 2 * U * (T + 64) * (np.abs(gz).T @ np.abs(X))
        err = np.abs(_f64(gw) - gw64)
        assert (err <= 1.01 * bound + 1e-35).all(), (err / (bound + 1e-35)).max()
    if gb is not None:
        if before is not None:
            gb64 = gb64 + before[1]
        bound = own.sum(axis=0) + 2 * U * (T + 64) * np.abs(gz).sum(axis=0) + U * np.abs(gb64)
        assert (np.abs(_f64(gb) - gb64) <= 1.01 * bound + 1e-35).all()


def both_ways(T, D, N, kind=b64.NONE, gated=False, pad=0, bias=None, residual=None, out=BF, seed=0, grad_w=F32, dy_pad=0, res_pad=0):
    b = gc.binding()
    x, W, bias_t, res = _draw(T, D, N, gated, pad, bias, residual, seed, res_pad)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    y, pre = b.rlf_linear_fwd(x, W, bias=bias_t, act=kind, gated=gated, residual=res, out_dtype=out, want_pre=True, dev_status=status)
    check_fwd(y, pre, x, W, bias_t, kind, gated, res)
    dy = (1e-2 * torch.randn(T, N + dy_pad, device=DEV)).to(out)[:, :N]
    args = dict(pre=pre, act=kind, gated=gated, grad_W_dtype=grad_w, want_grad_bias=True, dev_status=status)
    got = b.rlf_linear_bwd(dy, x, W, **args)
    check_bwd(got, dy, x, W, pre, kind, gated)
    for p, q in zip(got, b.rlf_linear_bwd(dy, x, W, **args)):
        assert torch.equal(p, q)
    assert status.item() == 0


SIZES = [(1, 8, 5), (1, 64, 128), (3, 2560, 130), (16, 264, 1000), (17, 128, 64), (65, 512, 257), (130, 1024, 96),
         (257, 72, 300), (300, 640, 5), (512, 128, 520), (1000, 320, 1031)]


@pytest.mark.parametrize("T,D,N", SIZES)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_sizes(T, D, N, gated):
    kind = ACTS[(T + N) % 5]
    both_ways(T, D, N, kind, gated, bias=BF)
    both_ways(T, D, N, b64.SILU, gated, pad=8, residual=BF, seed=1, grad_w=BF, dy_pad=3, res_pad=5)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("T,D,N,gated", [(5, 128, 200, False), (5, 128, 200, True), (400, 192, 136, False), (400, 192, 136, True)])
def test_activations(T, D, N, gated, kind):
    both_ways(T, D, N, kind, gated, bias=F32, residual=F32, out=F32)


@pytest.mark.parametrize("N", [1, 2, 3, 4])
@pytest.mark.parametrize("T,D", [(1, 8), (7, 64), (100, 2560), (5000, 136), (333, 4096), (9000, 24)])
def test_few_outputs(T, D, N):
    both_ways(T, D, N, bias=F32, out=F32, grad_w=BF)
    both_ways(T, D, N, ACTS[N], bias=BF, residual=BF, pad=16, seed=2, dy_pad=1)


@pytest.mark.parametrize("form,tile,split", [(1, 128, 0), (1, 256, 0), (2, 16, 1), (2, 32, 2), (2, 64, 4), (2, 128, 8), (2, 256, 2), (2, 256, 8), (2, 32, 3), (2, 64, 7), (1, 192, 0), (1, 64, 0), (3, 256, 0), (3, 128, 0)])
@pytest.mark.parametrize("T,D,N,gated", [(40, 512, 200, False), (40, 512, 200, True), (513, 328, 264, False), (300, 1024, 137, True)])
def test_every_form(form, tile, split, T, D, N, gated):
    b = gc.binding()
    b.tune_linear(form, tile, split)
    try:
        both_ways(T, D, N, b64.GELU, gated, bias=BF, residual=BF)
    finally:
        b.tune_linear()


def test_accumulation():
    b = gc.binding()
    for T, D, N in ((70, 256, 136), (600, 128, 264), (40, 64, 2)):
        x, W, _, _ = _draw(T, D, N)
        dy = torch.randn(T, N, device=DEV).to(BF)
        gw, gb = torch.randn(N, D, device=DEV), torch.randn(N, device=DEV)
        before = _f64(gw), _f64(gb)
        out = b.rlf_linear_bwd(dy, x, W, want_grad_x=False, grad_W=gw, grad_bias=gb, want_grad_bias=True, accumulate=True)
        assert out[0] is None and out[1] is gw and out[2] is gb
        check_bwd(out, dy, x, W, None, b64.NONE, False, before)


def test_no_rows_and_parts_of_the_gradient():
    b = gc.binding()
    x, W, _, _ = _draw(4, 64, 24)
    y, pre = b.rlf_linear_fwd(x[:0], W, act=b.ACT_SILU, want_pre=True)
    assert y.shape == (0, 24) and pre.shape == (0, 24)
    for n in (24, 3):
        g = torch.zeros(0, n, dtype=BF, device=DEV)
        gx, gw, gb = b.rlf_linear_bwd(g, x[:0], W[:n].contiguous(), want_grad_bias=True)
        assert gx.shape == (0, 64) and not gw.any() and not gb.any()
        gw += 3.0
        gb += 2.0
        b.rlf_linear_bwd(g, x[:0], W[:n].contiguous(), want_grad_x=False, grad_W=gw, grad_bias=gb, accumulate=True)
        assert (gw == 3).all() and (gb == 2).all()
    dy = torch.randn(4, 24, device=DEV).to(BF)
    full = b.rlf_linear_bwd(dy, x, W, want_grad_bias=True)
    for k in range(3):
        want = [k == i for i in range(3)]
        part = b.rlf_linear_bwd(dy, x, W, want_grad_x=want[0], want_grad_W=want[1], want_grad_bias=want[2])
        assert all((p is None) != w for p, w in zip(part, want)) and torch.equal(part[k], full[k])


def test_residual_in_place():
    b = gc.binding()
    for T, N, dt in ((9, 160, BF), (300, 264, BF), (300, 129, F32), (50, 2, F32)):
        x, W, _, res = _draw(T, 128, N, residual=dt)
        want, _ = b.rlf_linear_fwd(x, W, act=b.ACT_GELU, residual=res)
        got, _ = b.rlf_linear_fwd(x, W, act=b.ACT_GELU, residual=res, y_out=res)
        assert got is res and torch.equal(got, want)


def test_non_finite_inputs_stay_in_their_rows():
    b = gc.binding()
    for T, N in ((6, 96), (300, 264), (6, 3)):
        x, W, bias, _ = _draw(T, 128, N, bias=BF)
        clean, _ = b.rlf_linear_fwd(x, W, bias=bias, act=b.ACT_SILU)
        x[2, 5], x[4, 7], x[4, 9] = float("nan"), float("inf"), float("-inf")
        y, _ = b.rlf_linear_fwd(x, W, bias=bias, act=b.ACT_SILU)
        rest = [t for t in range(T) if t not in (2, 4)]
        assert torch.equal(y[rest], clean[rest]) and y[2].isnan().all()


def test_rows_behind_the_last_are_left_alone():
    b = gc.binding()
    for T, N in ((5, 72), (5, 71), (270, 136), (270, 135), (5, 2)):
        x, W, _, _ = _draw(T, 64, N)
        buf = torch.full((T + 40, N), 7.0, dtype=BF, device=DEV)
        pre = torch.full((T + 40, N), 7.0, dtype=BF, device=DEV)
        b.rlf_linear_fwd(x, W, act=b.ACT_RELU, y_out=buf[:T], pre_out=pre[:T])
        assert (buf[T:] == 7).all() and (pre[T:] == 7).all()
        gx = torch.full((T + 40, 64), 7.0, dtype=BF, device=DEV)
        gw = torch.full((N + 40, 64), 7.0, device=DEV)
        b.rlf_linear_bwd(buf[:T], x, W, pre=pre[:T], act=b.ACT_RELU, grad_x=gx[:T], grad_W=gw[:N])
        assert (gx[T:] == 7).all() and (gw[N:] == 7).all()


def test_gradient_against_differences():
    """sum(dy y) moved along a direction of x, W and bias, fp32 outputs (the outputs' own rounding would hide the slope)."""
    b = gc.binding()
    T, D, N, h = 12, 64, 40, 1.0 / 16
    for gated in (False, True):
        for kind in (b.ACT_SILU, b.ACT_GELU_TANH):
            x, W, bias, _ = _draw(T, D, N, gated, bias=F32)
            dy = torch.randn(T, N, device=DEV)
            f = lambda x_, W_, b_: (b.rlf_linear_fwd(x_, W_, bias=b_, act=kind, gated=gated, out_dtype=F32)[0].double() * dy.double()).sum().item()
            _, pre = b.rlf_linear_fwd(x, W, bias=bias, act=kind, gated=gated, want_pre=True)
            gx, gw, gb = b.rlf_linear_bwd(dy, x, W, pre=pre, act=kind, gated=gated, want_grad_bias=True)
            dirs = torch.randn_like(bias)
            num = (f(x, W, bias + h * dirs) - f(x, W, bias - h * dirs)) / (2 * h)
            ana = (gb.double() * dirs.double()).sum().item()
            scale = (gb.double() * dirs.double()).norm().item()
            # third derivatives of order one: h^2 / 6 of the terms' size, and bf16 pre-activations (2^-8)
            assert abs(num - ana) <= (h * h + 2.0 ** -7) * 8 * scale + 1e-3, (gated, kind, num, ana)


def test_other_stream_and_graph():
    b = gc.binding()
    x, W, bias, res = _draw(300, 192, 264, gated=True, bias=BF, residual=BF)
    dy = torch.randn(300, 264, device=DEV).to(BF)

    def step():
        y, pre = b.rlf_linear_fwd(x, W, bias=bias, act=b.ACT_SILU, gated=True, residual=res, want_pre=True)
        return (y, pre) + tuple(b.rlf_linear_bwd(dy, x, W, pre=pre, act=b.ACT_SILU, gated=True, want_grad_bias=True))

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    x.copy_(torch.randn_like(x))
    again = [t.clone() for t in step()]
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(kept, again))


def test_wrapper_refuses():
    b = gc.binding()
    x, W, bias, res = _draw(6, 64, 24, bias=BF, residual=BF)
    bad = [dict(x=x.float()), dict(W=W[:, :32].contiguous()), dict(W=W.t()), dict(bias=bias[:5]), dict(residual=res.float(), out_dtype=BF),
           dict(residual=res[:3]), dict(out_dtype=torch.float16), dict(x=x.cpu()), dict(gated=True, W=W[:23].contiguous()), dict(bias=bias.half())]
    for kw in bad:
        args = dict(x=x, W=W)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            b.rlf_linear_fwd(**args)
    dy = torch.randn(6, 24, device=DEV).to(BF)
    for kw in (dict(act=b.ACT_SILU), dict(grad_y=dy[:, :8]), dict(accumulate=True), dict(x=x.float()), dict(workspace=torch.empty(8, dtype=torch.uint8))):
        args = dict(grad_y=dy, x=x, W=W)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            b.rlf_linear_bwd(**args)
    for kw in (dict(x=torch.randn(6, 60, device=DEV).to(BF), W=torch.randn(8, 60, device=DEV).to(BF)), dict(act=9),
               dict(x=torch.randn(6, 67, device=DEV).to(BF)[:, :64])):
        args = dict(x=x, W=W)
        args.update(kw)
        with pytest.raises(b.RlfError):
            b.rlf_linear_fwd(**args)
    with pytest.raises(b.RlfError):
        b.rlf_linear_bwd(dy, x, W, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(b.RlfError):
        b.rlf_linear_bwd(dy, x, W, grad_W=torch.zeros(24, 64, dtype=BF, device=DEV), accumulate=True, want_grad_x=False)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("N,gated", [(2, False), (72, False), (71, False), (72, True), (71, True)])
def test_large_values_before_the_activation(N, gated, kind):
    """Finite values up to the type's largest, whose squares overflow fp32: z of column 0 is x's first element, every other
    column (and its part of W) is zero, the up half is one.  One term per sum, so an output is off by the activation's own error
    and its rounding, a gradient by those of the slope and of gz and itself to bf16."""
    b = gc.binding()
    big = [0.5, 3.0, 100.0, 3e4, 1e10, 6e19, 1e30, 3e38]
    x = torch.zeros(2 * len(big), 8, dtype=BF, device=DEV)
    x[:, 0] = torch.tensor(big + [-v for v in big])
    rows = 2 * N if gated else N
    W = torch.zeros(rows, 8, dtype=BF, device=DEV)
    W[0, 0] = 1.0
    bias = torch.zeros(rows, device=DEV)
    if gated:
        bias[N:] = 1.0
    y, pre = b.rlf_linear_fwd(x, W, bias=bias, act=kind, gated=gated, want_pre=True)
    z = _f64(x)[:, :1]
    small = np.minimum(np.abs(z), 100.0)        # (beyond that the slope is 0 or 1 to every digit)
    want = b64.act(z, kind)
    err = np.abs(_f64(y)[:, :1] - want)
    assert (err <= 1.01 * (2.0 ** -8 + _act_error(small, kind)) * np.abs(want) + 1e-30).all()
    dy = torch.ones(len(x), N, dtype=BF, device=DEV)
    gx, _, _ = b.rlf_linear_bwd(dy, x, W, pre=pre, act=kind, gated=gated, want_grad_W=False)
    slope = b64.act_grad(z, kind)
    bound = (_act_error(small, kind) + 8 * U) * (1 + small) + 2 * 2.0 ** -8 * np.abs(slope)
    err = np.abs(_f64(gx)[:, :1] - slope)
    assert (err <= 1.01 * bound).all()


@pytest.mark.parametrize("form,tile", [(0, 0), (1, 256), (1, 192), (1, 128), (1, 64), (3, 256), (3, 128)])
@pytest.mark.parametrize("T,D,N", [(700, 72, 328), (1100, 512, 1000), (257, 200, 72)])
def test_short_sums(form, tile, T, D, N):
    """Sums short enough that results leave 64 columns at a time (bf16, no `pre`, no residual), ragged in rows and columns; the
    gradients of a few tokens likewise, bf16 and fp32 ones in one launch too."""
    b = gc.binding()
    b.tune_linear(form, tile, 0)
    try:
        x, W, bias, _ = _draw(T, D, N, bias=BF)
        for kind in (b64.NONE, b64.SILU):
            buf = torch.full((T + 40, N), 7.0, dtype=BF, device=DEV)
            y, _ = b.rlf_linear_fwd(x, W, bias=bias, act=kind, y_out=buf[:T])
            check_fwd(y, None, x, W, bias, kind, False, None)
            assert (buf[T:] == 7).all()
        both_ways(T, D, N, grad_w=BF)
        both_ways(T, D, N)
        both_ways(200, D, N, grad_w=BF)
        both_ways(200, N // 8 * 8, D)
    finally:
        b.tune_linear(0, 0, 0)


@pytest.mark.parametrize("form", [0, 1, 2, 3])
@pytest.mark.parametrize("T,N,out,res_pad", [(300, 264, BF, 0), (300, 264, BF, 3), (300, 264, F32, 1), (130, 132, F32, 0), (130, 131, BF, 5), (130, 131, F32, 0)])
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_residual_and_output_on_any_boundary(form, T, N, out, res_pad, gated):
    """The residual's rows on 16-byte boundaries or not, its last columns fewer than a piece; output and `pre` aligned apart from
    each other."""
    b = gc.binding()
    b.tune_linear(form, 0, 0)
    try:
        both_ways(T, 200, N, b64.SILU, gated, bias=F32, residual=out, out=out, res_pad=res_pad)
    finally:
        b.tune_linear(0, 0, 0)
