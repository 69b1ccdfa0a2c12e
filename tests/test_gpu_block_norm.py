"""GPU parity of rlf_block_norm_fwd / rlf_block_norm_bwd against the fp64 definitions in oracle/blocks64.py.

Tolerances are error bounds, element by element, with u = 2^-24 (half a step of fp32), carried through the formulas:
  * a sum over a row is taken in chains of at most C = 96 additions (fast forms: 64 elements of a thread, 5 shuffles, 16
    warps; general form D / 256 + 13), so its error is at most C u sum |terms|;  1 / spread: half the relative error of its
    mean square plus 4 u (rsqrtf, the division by D), doubled for safety;  any other operation: u relative.
  * an error e of h moves the pre norm's input, its mean by at most mean e and its 1 / spread by r^2 mean |h - m| e relative.
  * a sum over tokens: chains of at most min(T, 700) + 164 additions.
  * the one rounding to the output's type: half a step (bf16 2^-8, fp32 2^-24).
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
EPS = 1e-5


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _half(dt):
    return 2.0 ** -8 if dt == BF else U


def _chain(D):
    return max(96, D // 256 + 16)


class Case:
    def __init__(self, T, D, dt=BF, w_dt=BF, post="rms", pre="rms", bias=False, form=None, alpha=1.0, beta=1.0, pad=0, seed=0, with_dh=True):
        self.__dict__.update(locals())
        g = torch.Generator(device=DEV)
        g.manual_seed(13 * seed + 5 * T + D)
        r = lambda *s: torch.randn(*s, generator=g, device=DEV)
        vec = lambda there, mean, spread: (mean + spread * r(D)).to(w_dt) if there else None
        self.x = (1.5 * r(T, D + pad) + 0.2).to(dt)[:, :D]
        self.residual = (2.0 * r(T, D) + 0.3).to(dt)
        self.w1, self.w2 = vec(post, 1.0, 0.3), vec(pre, 1.0, 0.3)
        self.b1, self.b2 = vec(post and bias, 0.0, 0.2), vec(pre and bias, 0.0, 0.2)
        self.gate = None if form is None else vec(True, 0.4, 0.5) if form == "column" else r(T)
        self.dy = (1e-2 * r(T, D)).to(dt) if pre else None
        self.dh = (1e-2 * r(T, D)).to(dt) if with_dh or not pre else None

    def kinds(self, b):
        k = {None: b.NORM_NONE, "rms": b.NORM_RMS, "layer": b.NORM_LAYER}
        return dict(post_kind=k[self.post], pre_kind=k[self.pre], gate=self.gate, alpha=self.alpha, beta=self.beta,
                    gate_form={None: b.GATE_NONE, "column": b.GATE_COLUMN, "row": b.GATE_ROW}[self.form])

    def forward(self, b, **kw):
        return b.rlf_block_norm_fwd(self.x, self.residual, post_weight=self.w1, post_bias=self.b1, pre_weight=self.w2, pre_bias=self.b2,
                                    eps=EPS, **self.kinds(b), **kw)

    def backward(self, b, h, stats, **kw):
        args = dict(post_weight=self.w1, post_bias=self.b1, pre_weight=self.w2, want_grad_bias=self.bias)
        args.update(self.kinds(b))
        args.update(kw)
        return b.rlf_block_norm_bwd(self.dy, self.dh, self.x, h, stats, **args)

    def spec(self):
        return dict(post=self.post, post_w=_f64(self.w1), post_b=_f64(self.b1), pre=self.pre, pre_w=_f64(self.w2), gate=_f64(self.gate),
                    form=self.form, alpha=self.alpha, beta=self.beta)

    def scale(self):
        g = _f64(self.gate)
        return np.abs(self.beta * (np.ones((1, 1)) if g is None else g[None, :] if self.form == "column" else g[:, None]))


def _unit_error(v, dv, kind, m, r, C):
    """errors of (v - m) r, of m and (relative) of r, from v known to dv"""
    if kind is None:
        return dv, np.zeros_like(m), np.zeros_like(r)
    dm = C * U * np.abs(v).mean(axis=1) + dv.mean(axis=1) if kind == "layer" else np.zeros_like(m)
    c = np.abs(v - m[:, None])
    # dm shifts the mean square by dm^2 only (the linear term cancels)
    dr = 2 * ((C / 2 + 4) * U + U * np.abs(v).max(axis=1) * r + 0.5 * (dm * r) ** 2 + r ** 2 * (c * dv).mean(axis=1))
    u = c * r[:, None]
    return r[:, None] * (dv + dm[:, None] + 2 * U * np.abs(v)) + u * (dr[:, None] + 4 * U), dm + U * np.abs(m), dr


def check_fwd(c, out):
    h, y, stats = out
    x, res = _f64(c.x), _f64(c.residual)
    h64, y64, s64 = b64.block_norm(x, res, pre_b=_f64(c.b2), eps=EPS, **c.spec())
    C, one = _chain(c.D), np.ones(c.D)
    w1, b1 = (np.abs(_f64(t)) if t is not None else k * one for t, k in ((c.w1, 1.0), (c.b1, 0.0)))
    du, dm, dr = _unit_error(x, np.zeros_like(x), c.post, s64[0], s64[1], C)
    n = np.abs((x - s64[0][:, None]) * s64[1][:, None]) * w1 + b1
    dh = c.scale() * (du * w1 + 6 * U * n) + 4 * U * (np.abs(c.alpha * res) + np.abs(h64))
    got = _f64(stats)
    assert (np.abs(got[0] - s64[0]) <= 1.01 * dm).all() and (np.abs(got[1] - s64[1]) <= 1.01 * dr * s64[1]).all()
    bound = dh + _half(c.dt) * np.abs(h64)
    err = np.abs(_f64(h) - h64)
    assert (err <= 1.01 * bound).all(), (err / bound).max()
    du, dm, dr = _unit_error(h64, dh, c.pre, s64[2], s64[3], C)
    assert (np.abs(got[2] - s64[2]) <= 1.01 * dm).all() and (np.abs(got[3] - s64[3]) <= 1.01 * dr * s64[3]).all()
    if c.pre is None:
        assert y is None
        return
    bound = du * np.abs(_f64(c.w2)) + 4 * U * (np.abs(y64) + (0 if c.b2 is None else np.abs(_f64(c.b2)))) + _half(c.dt) * np.abs(y64) + 1e-40
    err = np.abs(_f64(y) - y64)
    assert (err <= 1.01 * bound).all(), (err / bound).max()


def check_bwd(c, out, h, stats, before=None):
    x, H, s = _f64(c.x), _f64(h), _f64(stats)
    want = b64.block_norm_grad(_f64(c.dy), _f64(c.dh), x, H, s, **c.spec())
    C, one = _chain(c.D), np.ones(c.D)
    n_tok = min(c.T, 700) + 168
    m1, r1, m2, r2 = (v[:, None] for v in s)
    mean = lambda a: a.mean(axis=1, keepdims=True)
    gh = want["residual"] / c.alpha
    dgh = 4 * U * np.abs(gh) + (0 if c.dh is None else U * np.abs(_f64(c.dh)))
    if c.pre is not None:
        dy, u = np.abs(_f64(c.dy)), np.abs((H - m2) * r2)
        q = dy * np.abs(_f64(c.w2))
        a, b = mean(q * u), mean(q) if c.pre == "layer" else 0.0
        dgh = dgh + r2 * ((C + 8) * U * (b + u * a) + 8 * U * (q + u * a + b))
    s_abs, w1 = c.scale(), one if c.w1 is None else np.abs(_f64(c.w1))
    b1 = 0 * one if c.b1 is None else np.abs(_f64(c.b1))
    v = np.abs((x - m1) * r1)
    g, dg = s_abs * np.abs(gh) * w1, s_abs * w1 * dgh + 6 * U * s_abs * np.abs(gh) * w1
    bounds = dict(residual=abs(c.alpha) * dgh + (_half(c.dt) + 2 * U) * np.abs(want["residual"]))
    if c.post is None:
        bounds["x"] = dg + (_half(c.dt) + 4 * U) * np.abs(want["x"])
    else:
        a, b = mean(g * v), mean(g) if c.post == "layer" else 0.0
        da, db = mean(dg * v), mean(dg) if c.post == "layer" else 0.0
        bounds["x"] = r1 * (dg + db + v * da + (C + 8) * U * (b + v * a) + 8 * U * (g + v * a + b)) + (_half(c.dt) + 2 * U) * np.abs(want["x"])
    sgh, dsgh = s_abs * np.abs(gh), s_abs * dgh + 4 * U * s_abs * np.abs(gh)
    over = lambda d, terms: d.sum(axis=0) + n_tok * U * terms.sum(axis=0)
    e1, e2 = over(dsgh * v, sgh * v + 0 * v) + 8 * U * (sgh * v).sum(axis=0), over(dsgh, sgh)
    bounds.update(post_weight=e1, post_bias=e2)
    if c.pre is not None:
        bounds.update(pre_weight=(n_tok + 8) * U * (dy * u).sum(axis=0), pre_bias=n_tok * U * dy.sum(axis=0))
    if c.form is not None:
        n = v * w1 + b1
        terms, d = abs(c.beta) * np.abs(gh) * n, abs(c.beta) * (dgh + 8 * U * np.abs(gh)) * n
        bounds["gate"] = over(d, terms) + 8 * U * terms.sum(axis=0) if c.form == "column" else d.sum(axis=1) + (C + 16) * U * terms.sum(axis=1)
    for k, w in want.items():
        t = out["grad_" + k]
        if t is None:
            continue
        if before is not None and k in before:
            w = w + before[k]
            bounds[k] = bounds[k] + U * np.abs(w)
        err, bound = np.abs(_f64(t) - w), 1.01 * bounds[k] + 1e-40
        assert (err <= bound).all(), (k, (err / bound).max())


def both_ways(*a, **kw):
    b = gc.binding()
    c = Case(*a, **kw)
    out = c.forward(b)
    check_fwd(c, out)
    got = c.backward(b, out[0], out[2])
    check_bwd(c, got, out[0], out[2])
    again = c.backward(b, out[0], out[2])
    for k, t in got.items():
        assert (t is None and again[k] is None) or torch.equal(t, again[k]), k
    return c, out, got


SIZES = [(1, 1), (1, 64), (3, 7), (5, 1021), (2, 31), (17, 2560), (64, 4096), (9, 8192), (2, 16384), (3, 20001), (300, 512), (4097, 128),
         (33, 2604), (1030, 1022), (700, 5120)]


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("dt,w_dt", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_sizes(T, D, dt, w_dt, kind):
    both_ways(T, D, dt, w_dt, kind, kind)
    both_ways(T, D, dt, w_dt, kind, kind, bias=True, form="column", alpha=0.75, beta=0.5, pad=8, seed=1)
    both_ways(T, D, dt, w_dt, kind, kind, form="row", beta=-1.5, pad=3, seed=2, with_dh=False)


@pytest.mark.parametrize("post,pre", [("rms", None), (None, "rms"), ("layer", None), (None, "layer"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("form", [None, "column", "row"])
@pytest.mark.parametrize("T,D,dt,pad", [(70, 768, BF, 0), (70, 768, BF, 3), (41, 333, F32, 0), (41, 333, BF, 1)])
def test_norms_and_gates(T, D, dt, pad, form, post, pre):
    both_ways(T, D, dt, F32, post, pre, bias=True, form=form, alpha=1.25, beta=0.5, pad=pad)
    both_ways(T, D, dt, BF, post, pre, bias=False, form=form, pad=pad, seed=3, with_dh=False)


def test_residual_in_place_and_slices_off_their_vectors():
    b = gc.binding()
    for T, D, dt in ((50, 512, BF), (50, 515, F32), (7, 8200, BF)):
        c = Case(T, D, dt, F32, "rms", "layer", form="row")
        want = c.forward(b)
        got = c.forward(b, h_out=c.residual)
        assert got[0] is c.residual and all(torch.equal(p, q) for p, q in zip(got, want))
        c = Case(T, D, dt, F32, "layer", "rms", bias=True, form="column")
        # every tensor one element behind a 16-byte boundary, and each somewhere else in its vector
        for shifts in ((1,) * 6, (1, 2, 3, 0, 1, 2)):
            def at(t, k):
                buf = torch.full((t.numel() + 16,), float("nan"), dtype=t.dtype, device=DEV)
                out = buf[k:k + t.numel()].view(t.shape)
                out.copy_(t)
                return out
            c.x, c.residual, c.dy, c.dh = (at(t.contiguous(), k) for t, k in zip((c.x, c.residual, c.dy, c.dh), shifts))
            y, h = at(c.dy, shifts[4]), at(c.dy, shifts[5])
            out = c.forward(b, y_out=y, h_out=h)
            check_fwd(c, out)
            check_bwd(c, c.backward(b, h, out[2], grad_x=at(c.dy, shifts[2]), grad_residual=at(c.dy, shifts[1])), h, out[2])


def test_accumulation_and_parts():
    b = gc.binding()
    for D, pad in ((256, 0), (259, 2)):
        c = Case(90, D, BF, BF, "layer", "rms", bias=True, form="column", pad=pad)
        h, _, stats = c.forward(b)
        names = ["post_weight", "post_bias", "pre_weight", "pre_bias", "gate"]
        bufs = {k: torch.randn(D, device=DEV) for k in names}
        before = {k: _f64(t) for k, t in bufs.items()}
        out = c.backward(b, h, stats, accumulate=True, **{"grad_" + k: t for k, t in bufs.items()})
        check_bwd(c, out, h, stats, before)
        full = c.backward(b, h, stats)
        off = dict(want_grad_x=False, want_grad_residual=False, want_grad_weight=False, want_grad_bias=False, want_grad_gate=False)
        flag = dict(grad_x="want_grad_x", grad_residual="want_grad_residual", grad_gate="want_grad_gate", grad_post_bias="want_grad_bias",
                    grad_pre_weight="want_grad_weight")
        for k, f in flag.items():
            part = c.backward(b, h, stats, **dict(off, **{f: True}))
            assert torch.equal(part[k], full[k]), k
            assert all(v is None for n, v in part.items() if n != k and not ("weight" in n and "weight" in k) and not ("bias" in n and "bias" in k))
        c = Case(90, D, BF, BF, "rms", "rms", form="row", pad=pad)
        h, _, stats = c.forward(b)
        only = c.backward(b, h, stats, **dict(off, want_grad_gate=True))
        assert torch.equal(only["grad_gate"], c.backward(b, h, stats)["grad_gate"])


def test_no_rows():
    b = gc.binding()
    c = Case(4, 64, form="column")
    c.x, c.residual, c.dy, c.dh, c.T = c.x[:0], c.residual[:0], c.dy[:0], c.dh[:0], 0
    h, y, stats = c.forward(b)
    assert h.shape == (0, 64) and y.shape == (0, 64) and stats.shape == (4, 0)
    g = c.backward(b, h, stats)
    assert not g["grad_post_weight"].any() and not g["grad_pre_weight"].any() and not g["grad_gate"].any()
    g["grad_gate"] += 2
    c.backward(b, h, stats, accumulate=True, **g)
    assert (g["grad_gate"] == 2).all()


def test_non_finite_rows_stay_alone():
    b = gc.binding()
    for D, pad in ((512, 0), (509, 0), (512, 3)):
        c = Case(40, D, BF, BF, "layer", "rms", bias=True, form="column", pad=pad)
        h, y, stats = c.forward(b)
        clean = c.backward(b, h, stats)
        rest = [t for t in range(40) if t not in (3, 17, 39)]
        c.x[3, 5], c.residual[17, 0], c.x[39, D - 1] = float("nan"), float("inf"), float("-inf")
        h2, y2, stats2 = c.forward(b)
        assert torch.equal(h2[rest], h[rest]) and torch.equal(y2[rest], y[rest]) and torch.equal(stats2[:, rest], stats[:, rest])
        assert h2[3].isnan().all() and y2[17].isnan().any() and h2[39].isnan().any()
        g = c.backward(b, h2, stats2)
        assert torch.equal(g["grad_x"][rest], clean["grad_x"][rest]) and torch.equal(g["grad_residual"][rest], clean["grad_residual"][rest])


def test_rows_behind_the_last_are_left_alone():
    b = gc.binding()
    for D in (256, 261):
        c = Case(6, D, BF, F32, "rms", "rms", form="row")
        buf = lambda: torch.full((30, D), 7.0, dtype=BF, device=DEV)
        h, y, gx, gr = buf(), buf(), buf(), buf()
        out = c.forward(b, h_out=h[:6], y_out=y[:6])
        gate = torch.full((30,), 7.0, device=DEV)
        c.backward(b, h[:6], out[2], grad_x=gx[:6], grad_residual=gr[:6], grad_gate=gate[:6])
        assert all((t[6:] == 7).all() for t in (h, y, gx, gr, gate))


def test_gradient_against_differences():
    """Directional differences of sum(dy y) + sum(dh h), fp32 rows, along x, the residual, the weights and the gate."""
    b = gc.binding()
    for post, pre in (("layer", "rms"), ("rms", "layer")):
        for form in ("column", "row"):
            c = Case(5, 96, F32, F32, post, pre, bias=True, form=form, alpha=0.75, beta=1.25)
            h, _, stats = c.forward(b)
            g = c.backward(b, h, stats)
            slots = dict(x="grad_x", residual="grad_residual", w1="grad_post_weight", w2="grad_pre_weight", b1="grad_post_bias",
                         b2="grad_pre_bias", gate="grad_gate")

            def total():
                h_, y_, _ = c.forward(b)
                return (c.dy.double() * y_.double()).sum().item() + (c.dh.double() * h_.double()).sum().item()

            for name, key in slots.items():
                t = getattr(c, name)
                kept, d, e = t.clone(), torch.randn_like(t), 1.0 / 64
                t.copy_(kept + e * d)
                up = total()
                t.copy_(kept - e * d)
                down = total()
                t.copy_(kept)
                terms = g[key].double() * d.double()
                # the difference's own error: e^2 / 6 of third derivatives of the terms' size, and outputs to 2^-22 over 2 e
                bound = 8 * e * e * terms.norm().item() * 4 + 2.0 ** -22 / (2 * e) * 2 * (c.dy.double().abs().sum().item() * 3)
                assert abs((up - down) / (2 * e) - terms.sum().item()) <= bound, (post, pre, form, name)


def test_other_stream_and_graph():
    b = gc.binding()
    c = Case(200, 640, BF, F32, "layer", "rms", bias=True, form="column")

    def step():
        h, y, stats = c.forward(b)
        return [h, y, stats] + list(c.backward(b, h, stats).values())

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
    c.x.copy_(torch.randn_like(c.x))
    again = [t.clone() for t in step()]
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(kept, again))


def test_wrapper_refuses():
    b = gc.binding()
    c = Case(6, 64, BF, BF, "rms", "rms", form="column")
    h, y, stats = c.forward(b)
    good = dict(post_weight=c.w1, pre_weight=c.w2, gate=c.gate, gate_form=b.GATE_COLUMN)
    for kw in (dict(post_weight=None), dict(pre_weight=c.w2.float()), dict(gate=None), dict(gate_form=b.GATE_NONE), dict(gate=c.gate[:5]),
               dict(gate_form=b.GATE_ROW), dict(post_kind=b.NORM_NONE), dict(residual=c.residual.float()), dict(residual=c.residual[:3]),
               dict(x=c.x.half()), dict(x=c.x.cpu()), dict(x=c.x.t()), dict(y_out=y[:2])):
        args = dict(x=c.x, residual=c.residual, **good)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            b.rlf_block_norm_fwd(**args)
    for kw in (dict(grad_y=None), dict(h=None), dict(stats=stats[:2]), dict(accumulate=True), dict(grad_x=h.float())):
        args = dict(grad_y=c.dy, grad_h=c.dh, x=c.x, h=h, stats=stats, **good)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            b.rlf_block_norm_bwd(**args)
    for kw in (dict(eps=0.0), dict(alpha=float("nan")), dict(beta=float("inf")), dict(post_kind=7)):
        args = dict(x=c.x, residual=c.residual, **good)
        args.update(kw)
        with pytest.raises(b.RlfError):
            b.rlf_block_norm_fwd(**args)
    with pytest.raises(b.RlfError):
        b.rlf_block_norm_fwd(c.x, c.residual, post_kind=b.NORM_NONE, pre_kind=b.NORM_NONE)
    with pytest.raises(b.RlfError):
        b.rlf_block_norm_bwd(c.dy, c.dh, c.x, h, stats, workspace=torch.empty(256, dtype=torch.uint8, device=DEV), **good)


@pytest.mark.parametrize("T,D,dt", [(400, 7104, F32), (400, 6001, F32), (350, 8188, F32), (330, 5600, F32), (6000, 72, BF), (6000, 40, F32)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_long_rows_and_many_partial_rows(T, D, dt, kind):
    """fp32 rows too long for two buffers, several to a CTA; narrow rows, whose partial sums a cluster of CTAs adds up."""
    both_ways(T, D, dt, F32, kind, kind, bias=kind == "layer", form="column", alpha=0.75, beta=0.5)
    both_ways(T, D, dt, dt, kind, kind, form="row", pad=3, seed=1, with_dh=False)
