"""GPU parity of rlf_fused_lmhead_cross_entropy against the fp64 definition in oracle/operators64.py.

Tolerances are error bounds, u = 2^-24, h = 2^-8 (half a step of bf16), "acc(K)" = (K / 8 + 16) 2^-23 for a
tensor-core sum of K products (at least eight products per accumulation step, each step off by less than one
fp32 step whatever its rounding):
  * a logit: dz = acc(D) max_v sum_d |h_d W_vd|;  lse and the log-prob: dz + u (|M| + |rho| + 2 E(M - z) + 3 |lse| + 340)
    + 2^-22 (256 terms per thread and tile, 64 partials, the reference rho up to |z_y| + 32 away);
  * an entry of grad_z: that, plus the exponential's own u (|M| + |rho| + 2 (M - z) + 40) + 2^-21 relative, plus one
    rounding to bf16 (h) of the stored exponential; in grad_W one more rounding (h) of the scaled hidden row;
  * the products: the entries' errors times |W| (|hidden|) summed, acc(V) (acc(T)) of the sum of magnitudes, and the
    rounding of the result (h or u); the smoothing vectors: sums of at most V / 32 + 200 terms.
"""
import numpy as np
import pytest
import torch

from oracle import operators64 as o64
import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, HB = 2.0 ** -24, 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(params=["pair2", "pair1", "single", "universal"])
def form(request):
    """The forms of the contraction kernel: CTA pairs with two or one accumulators in the gradients, single CTAs, and
    the scratch that holds dZ itself from the start."""
    b = gc.binding()
    b.tune_lmhead(0 if request.param == "single" else 1)
    b.tune_lmhead_backward(0 if request.param == "universal" else 1, 0 if request.param == "pair1" else 1)
    yield request.param
    b.tune_lmhead(1)
    b.tune_lmhead_backward(1, 1)


def _inputs(T, D, V, seed, w_std=None, live=0.7):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    H = torch.randn(T, D, generator=g, device=DEV).to(BF)
    W = (torch.randn(V, D, generator=g, device=DEV) * (w_std or 2.0 / D ** 0.5)).to(BF)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    mask = (torch.rand(T, generator=g, device=DEV) < live).to(torch.uint8)
    mask[T // 2] = 1
    # a few targets that the model is nearly sure of
    for t in range(0, T, 5):
        H[t] = (H[t].float() + 0.6 * D ** 0.5 * W[ids[t].long()].float() / W[ids[t].long()].float().norm()).to(BF)
    return H, W, ids, mask


def run(H, W, ids, mask, eps=0.0, zc=0.0, status=0, **kw):
    b = gc.binding()
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = b.rlf_fused_lmhead_cross_entropy(H, W, ids, mask, label_smoothing=eps, z_coef=zc, dev_status=st, **kw)
    assert st.item() == status, st.item()
    return out


def check(out, H, W, ids, mask, eps=0.0, zc=0.0, denom=None, gw0=None):
    logp, lse, loss, gh, gw = out
    H64, W64 = (t.double().cpu().numpy() for t in (H, W))
    H64 = np.where(np.isfinite(H64), H64, np.nan)
    y = ids.cpu().numpy()
    m = None if mask is None else mask.cpu().numpy()
    with np.errstate(all="ignore"):
        r = o64.fused_cross_entropy(H64, W64, y, m, eps, zc, denom)
    live = np.flatnonzero(r["live"])
    T, D = H64.shape
    V = W64.shape[0]
    lp = logp.double().cpu().numpy()
    assert np.array_equal(np.isnan(lp), ~r["live"])
    if live.size == 0:
        assert not loss.any() and (gh is None or not gh.any()) and (gw is None or not gw.any())
        return r
    Hl = H64[live]
    z = Hl @ W64.T
    M = z.max(axis=1, keepdims=True)
    p = np.exp(z - r["lse"][live][:, None])
    acc = lambda K: (K / 8 + 16) * 2.0 ** -23
    dz = (acc(D) * (np.abs(Hl) @ np.abs(W64).T).max(axis=1))[:, None]
    zy = z[np.arange(live.size), y[live]][:, None]
    rho = np.abs(zy) + 32
    l = np.abs(r["lse"][live])[:, None]
    dl = dz + U * (np.abs(M) + rho + 2 * (p * (M - z)).sum(axis=1, keepdims=True) + 3 * l + 340) + 2.0 ** -22
    assert (np.abs(lp[live] - r["logp"][live]) <= (2 * dl[:, 0] + 3 * U * np.abs(r["logp"][live]))).all()
    if lse is not None:
        assert (np.abs(lse.double().cpu().numpy()[live] - r["lse"][live]) <= dl[:, 0]).all()
    absu = np.abs(W64).sum(axis=0)
    mean_err = dz[:, 0] + (V / 32 + 200) * U * (np.abs(Hl) @ absu) / V + 4 * U * (l + np.abs(M))[:, 0]
    tol = [0, (2 * dl[:, 0] + 3 * U * np.abs(r["logp"][live])).sum(), (dl[:, 0] + mean_err).sum() if eps else 0.0,
           ((2 * l + 1) * (dl + U * l)).sum()]
    tol[0] = tol[1] + eps * tol[2] + zc * tol[3]
    for k in range(4):
        assert abs(loss[k].item() - r["loss"][k]) <= tol[k] / r["n"] + 1e-12 * abs(r["loss"][k]), k
    if gh is None and gw is None:
        return r
    c = 1.0 / r["n"]
    A = np.abs(1 + 2 * zc * r["lse"][live])[:, None]
    rel = 2 * dl + dz + U * (np.abs(M) + rho + 2 * (M - z) + 40) + 2.0 ** -21 + 2 * zc * dl
    err = c * A * p * (rel + 1.01 * HB)
    g64 = r["grad"][live] + c * eps / V                    # what the scratch stands for: without the uniform part
    at = (np.arange(live.size), y[live])
    # the target entry: formed in fp32 from the log-prob, then rounded once
    err[at] = (np.abs(g64[at]) * 1.01 * HB + c * (2 * dl[:, 0] * np.minimum(1.0, 2 * p[at]) + 2 * zc * l[:, 0] * p[at] * (2 * dl[:, 0] + 8 * U)
               + 8 * U * (eps + np.abs(g64[at]) / c) + 4 * U * np.abs(zy[:, 0]) * p[at]))
    # the scratch holds exp(z - rho), rho = z_y + 32, and drops what is below the normal range (2^-126); the row's factor is
    # c A exp(rho - lse) <= c A e^32 since z_y <= lse: entries of grad_z below c A 1e-24 may be lost (the universal form's
    # references are tile maxima, its factor at most c A)
    tiny = c * A * 2.0 ** -126 * np.exp(32.0)
    err = err + tiny
    mag = np.abs(g64) + err
    absW, absH = np.abs(W64), np.abs(Hl)
    if gh is not None:
        got = gh.double().cpu().numpy()
        assert not got[~r["live"]].any()
        want = r["grad_hidden"][live]
        bound = err @ absW + acc(V) * (mag @ absW) + c * eps / V * (V / 32 + 210) * U * absu + 1.01 * HB * np.abs(want)
        e = np.abs(got[live] - want)
        assert (e <= bound).all(), (e / bound).max()
    if gw is not None:
        got = gw.double().cpu().numpy() - (0.0 if gw0 is None else gw0.double().cpu().numpy())
        half = 1.01 * HB if gw.dtype == BF else 2 * U
        want = r["grad_W"]
        bound = ((err + 1.01 * HB * mag).T @ absH + acc(T) * (mag.T @ absH) + c * eps / V * (T / 32 + 210) * U * absH.sum(axis=0)
                 + half * np.abs(want) + (0.0 if gw0 is None else 2 * U * (np.abs(gw0.double().cpu().numpy()) + np.abs(want))))
        e = np.abs(got - want)
        assert (e <= bound).all(), (e / bound).max()
    return r


@pytest.mark.parametrize("T,D,V", [(320, 128, 2048), (1, 64, 8), (130, 64, 1032), (257, 320, 4360), (7, 192, 520), (64, 2560, 3000)])
def test_sizes_and_objectives(T, D, V, form):
    H, W, ids, mask = _inputs(T, D, V, T + D)
    for eps, zc in ((0.0, 0.0), (0.1, 0.0), (0.0, 1e-3), (0.2, 1e-2)):
        check(run(H, W, ids, mask, eps, zc), H, W, ids, mask, eps, zc)
        check(run(H, W, ids, mask, eps, zc, grad_W_dtype=BF), H, W, ids, mask, eps, zc)
        check(run(H, W, ids, mask, eps, zc, want_grad_hidden=False, want_grad_W=False), H, W, ids, mask, eps, zc)
    check(run(H, W, ids, None, 0.1), H, W, ids, None, 0.1)


def test_full_vocabulary():
    H, W, ids, mask = _inputs(300, 256, 151936, 3)
    for eps in (0.0, 0.1):
        check(run(H, W, ids, mask, eps, 1e-4, grad_W_dtype=BF), H, W, ids, mask, eps, 1e-4)


@pytest.mark.parametrize("D", [64, 2560])
def test_few_tokens_of_a_wide_head(D):
    """One to a few dozen rows against a long vocabulary (the long axis of grad_hidden is the vocabulary)."""
    for T in (1, 2, 33, 64, 129):
        H, W, ids, mask = _inputs(T, D, 20008, T, live=0.9)
        check(run(H, W, ids, mask, 0.1, 1e-4, grad_W_dtype=BF), H, W, ids, mask, 0.1, 1e-4)
        check(run(H, W, ids, mask), H, W, ids, mask)


def test_partial_outputs_agree(form):
    H, W, ids, mask = _inputs(200, 128, 1000, 4)
    full = run(H, W, ids, mask, 0.1, 1e-3)
    a = run(H, W, ids, mask, 0.1, 1e-3, want_grad_W=False, want_lse=False)
    b = run(H, W, ids, mask, 0.1, 1e-3, want_grad_hidden=False)
    assert a[1] is None and a[4] is None and b[3] is None
    assert torch.equal(a[3], full[3]) and torch.equal(b[4], full[4]) and torch.equal(a[2], full[2])


def test_masks_targets_and_no_rows(form):
    b = gc.binding()
    H, W, ids, mask = _inputs(150, 64, 776, 5)
    none = torch.zeros_like(mask)
    out = run(H, W, ids, none, 0.1, 1e-4)
    check(out, H, W, ids, none, 0.1, 1e-4)
    out = run(H, W, ids, none, 0.1, 1e-4, grad_W_dtype=BF)
    assert not out[4].any() and not out[3].any() and not out[2].any()
    ids2 = ids.clone()
    ids2[mask == 0] = -100
    check(run(H, W, ids2, mask, 0.1), H, W, ids2, mask, 0.1)
    bad = torch.nonzero(mask).flatten()[:2]
    ids2[bad[0]], ids2[bad[1]] = 776, -5
    r = check(run(H, W, ids2, mask, 0.1, status=b.DEV_BAD_TARGET), H, W, ids2, mask, 0.1)
    assert r["n"] == int((mask != 0).sum())
    gw0 = torch.randn(776, 64, device=DEV)
    keep = gw0.clone()
    e = run(H[:0], W, ids[:0], mask[:0], grad_W=gw0, accumulate_grad_W=True)
    assert torch.equal(gw0, keep) and not e[2].any() and e[3].shape == (0, 64)
    for dt in (BF, F32):
        assert not run(H[:0], W, ids[:0], None, grad_W=torch.ones(776, 64, device=DEV, dtype=dt))[4].any()


def test_a_non_finite_row_is_taken_out_alone(form):
    b = gc.binding()
    H, W, ids, mask = _inputs(140, 64, 1032, 6)
    mask[3] = mask[77] = 1
    mask[10] = 0
    H[10] = float("nan")                          # not looked at: the row carries no loss
    check(run(H, W, ids, mask, 0.1), H, W, ids, mask, 0.1)
    H[3, 5] = float("nan")
    H[77, 0] = float("inf")
    for dt in (BF, F32):
        out = run(H, W, ids, mask, 0.1, status=b.DEV_NONFINITE, grad_W_dtype=dt)
        r = check(out, H, W, ids, mask, 0.1)
        assert not r["live"][[3, 77]].any() and torch.isfinite(out[4]).all() and torch.isfinite(out[3]).all()


@pytest.mark.parametrize("T", [5, 300])
def test_a_head_with_a_non_finite_row_gives_zero_gradients(form, T):
    """Every row's logits hold a NaN (or, with smoothing, an infinite mean): all rows are taken out, gradients zeros."""
    b = gc.binding()
    H, W, ids, mask = _inputs(T, 64, 1032, 12)
    H = H.abs() + 1.0
    for bad, eps in ((float("nan"), 0.0), (float("nan"), 0.1), (float("-inf"), 0.1), (float("inf"), 0.0)):
        W[5, 7] = bad
        for dt in (BF, F32):
            lp, lse, _, gh, gw = run(H, W, ids, mask, eps, status=b.DEV_NONFINITE, grad_W_dtype=dt)
            assert torch.isnan(lp).all() and torch.isnan(lse).all()
            assert not gh.any() and not gw.any()


def test_targets_far_below_the_maximum_take_the_universal_scratch():
    """A target 130 below its row's maximum lies outside the window of the per-row reference: its chunk is redone,
    with the universal form's bits."""
    b = gc.binding()
    H, W, ids, mask = _inputs(200, 64, 1032, 7)
    t = int(torch.nonzero(mask).flatten()[5])
    w = W[ids[t].long()].float()
    H[t] = (-130.0 * w / (w * w).sum()).to(BF)
    far = [run(H, W, ids, mask, 0.1, 1e-3, grad_W_dtype=dt) for dt in (BF, F32)]
    for o in far:
        check(o, H, W, ids, mask, 0.1, 1e-3)
    assert far[0][0][t].item() < -100
    b.tune_lmhead_backward(0, 1)
    try:
        ref = run(H, W, ids, mask, 0.1, 1e-3)
    finally:
        b.tune_lmhead_backward(1, 1)
    assert torch.equal(ref[3], far[1][3]) and torch.equal(ref[4], far[1][4])


def test_z_loss_that_cancels_the_softmax_part(form):
    """1 + 2 zeta lse near zero or negative: all logits around -16, zeta 0.05."""
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    H = (1.0 + 0.1 * torch.randn(60, 64, generator=g, device=DEV)).to(BF)
    W = (-0.25 + 0.02 * torch.randn(504, 64, generator=g, device=DEV)).to(BF)
    ids = torch.randint(0, 504, (60,), generator=g, device=DEV, dtype=torch.int32)
    for zc in (0.05, 0.2):
        check(run(H, W, ids, None, 0.0, zc), H, W, ids, None, 0.0, zc)
        check(run(H, W, ids, None, 0.1, zc, grad_W_dtype=BF), H, W, ids, None, 0.1, zc)


def test_several_chunks_and_accumulation():
    """More tokens than one chunk of the scratch holds (18944), with the last chunks free of live rows or not."""
    T = 18944 * 2 + 100
    H, W, ids, mask = _inputs(T, 64, 264, 9, live=0.9)
    for tail_dead in (False, True):
        if tail_dead:
            mask[9000:] = 0
        check(run(H, W, ids, mask, 0.1, 1e-3, grad_W_dtype=BF), H, W, ids, mask, 0.1, 1e-3)
        gw0 = torch.randn(264, 64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) * 1e-3
        out = run(H, W, ids, mask, 0.1, 1e-3, grad_W=gw0.clone(), accumulate_grad_W=True)
        check(out, H, W, ids, mask, 0.1, 1e-3, gw0=gw0)
    b = gc.binding()
    H, W, ids, mask = _inputs(1500, 128, 1032, 10)
    b.tune_lmhead_schedule(0, 0, 4)
    try:
        check(run(H, W, ids, mask, 0.1), H, W, ids, mask, 0.1)
        check(run(H, W, ids, mask, 0.1, grad_W_dtype=BF), H, W, ids, mask, 0.1)
    finally:
        b.tune_lmhead_schedule(0, 0, 0)


def test_micro_batches_against_a_common_count_add_up():
    H, W, ids, mask = _inputs(300, 128, 1032, 11)
    n = (mask != 0).sum().reshape(1)
    whole = run(H, W, ids, mask, 0.1, 1e-3)
    gw = torch.zeros(1032, 128, device=DEV)
    loss = 0.0
    for a, z in ((0, 100), (100, 101), (101, 300)):
        o = run(H[a:z], W, ids[a:z], mask[a:z], 0.1, 1e-3, denom=n, grad_W=gw, accumulate_grad_W=True)
        loss = loss + o[2]
        assert (o[3].double() - whole[3][a:z].double()).abs().max() <= 2.0 ** -7 * whole[3].double().abs().max()
    assert torch.allclose(loss, whole[2], rtol=1e-6)
    check((whole[0], whole[1], whole[2], whole[3], gw), H, W, ids, mask, 0.1, 1e-3)


def test_refusals():
    b = gc.binding()
    H, W, ids, mask = _inputs(8, 64, 64, 12)
    with pytest.raises(b.RlfError) as e:
        run(H, W, ids, mask, grad_W=torch.zeros(64, 64, dtype=BF, device=DEV), accumulate_grad_W=True)
    assert e.value.code == -8
    with pytest.raises(ValueError):
        run(H, W, ids, mask, accumulate_grad_W=True)
    with pytest.raises(TypeError):
        run(H, W.float(), ids, mask)
    with pytest.raises(b.RlfError):
        run(H, W[:63].contiguous(), ids, mask)
    with pytest.raises(ValueError):
        run(H.t(), W, ids, mask)


def test_gradient_against_differences():
    """Central differences of the call's own fp64 loss along one entry of the hidden state and of the head (steps that
    bf16 holds exactly).  Truncation: h^2 / 6 times a third derivative of at most the cube of the other factor's
    largest entry; rounding: 2^-21 (|lse| < 8) per loss term over h."""
    g = torch.Generator(device=DEV)
    g.manual_seed(13)
    q = lambda t: (torch.round(t * 16) / 16).to(BF)
    H, W = q(torch.randn(5, 64, generator=g, device=DEV)), q(0.25 * torch.randn(40, 64, generator=g, device=DEV))
    ids = torch.randint(0, 40, (5,), generator=g, device=DEV, dtype=torch.int32)
    eps, zc, h = 0.1, 1e-2, 2.0 ** -4
    _, _, _, gh, gw = run(H, W, ids, None, eps, zc)
    gh, gw = gh.clone(), gw.clone()
    f = lambda a, b: run(a, b, ids, None, eps, zc)[2][0].item()
    for (t, d) in ((0, 0), (4, 63)):
        e = torch.zeros_like(H)
        e[t, d] = h
        fd = (f(H + e, W) - f(H - e, W)) / (2 * h)
        tol = h * h / 6 * 2 * W.float().abs().max().item() ** 3 / 5 + 2.0 ** -21 / h + 2 * HB * gh.float().abs().max().item()
        assert abs(fd - gh[t, d].item()) <= tol, (fd, gh[t, d].item(), tol)
    for (v, d) in ((int(ids[0]), 3), (7, 60)):
        e = torch.zeros_like(W)
        e[v, d] = h
        fd = (f(H, W + e) - f(H, W - e)) / (2 * h)
        tol = h * h / 6 * 2 * H.float().abs().max().item() ** 3 + 2.0 ** -21 / h + 3 * HB * gw.abs().max().item()
        assert abs(fd - gw[v, d].item()) <= tol, (fd, gw[v, d].item(), tol)


def test_repeated_captured_and_on_another_stream():
    H, W, ids, mask = _inputs(500, 256, 4360, 14)
    b = gc.binding()
    call = lambda: b.rlf_fused_lmhead_cross_entropy(H, W, ids, mask, label_smoothing=0.1, z_coef=1e-4, grad_W_dtype=BF)
    ref = call()
    same = lambda o: all(torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in zip(o, ref))
    for _ in range(3):
        assert same(call())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert same(o)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    H0, ids0, mask0 = H.clone(), ids.clone(), mask.clone()
    H.copy_(H0.flip(0)), ids.copy_(ids0.flip(0)), mask.copy_(mask0.flip(0))
    g.replay()
    torch.cuda.synchronize()
    check(out, H, W, ids, mask, 0.1, 1e-4)
    H.copy_(H0), ids.copy_(ids0), mask.copy_(mask0)
    g.replay()
    torch.cuda.synchronize()
    assert same(out)


def test_agrees_with_the_logits_form():
    b = gc.binding()
    H, W, ids, mask = _inputs(256, 512, 8008, 15)
    z = H.float() @ W.float().t()
    a = run(H, W, ids, mask, 0.1, 1e-3)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    c = b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=0.1, z_coef=1e-3, dev_status=st)
    live = mask != 0
    assert (a[0][live] - c[0][live]).abs().max() <= 1e-4 and torch.allclose(a[2], c[2], rtol=1e-5)
    gh, gw = c[3] @ W.float(), c[3].t() @ H.float()
    assert (a[3].float() - gh).abs().max() <= 2.0 ** -6 * gh.abs().max()
    assert (a[4] - gw).abs().max() <= 2.0 ** -6 * gw.abs().max()
