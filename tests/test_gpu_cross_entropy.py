"""GPU parity of rlf_cross_entropy_fwd_bwd against the fp64 definition in oracle/operators64.py.

Tolerances are error bounds per row, u = 2^-24 (half a step of fp32), M the row's maximum, E = sum_v p_v:
  * an exponential: its exponent is formed with an error of at most u (|M| + 2 (M - z)) (rounding of M log2 e,
    of log2 e itself, and of the result), the exponential itself with 2^-22 relative;
  * the sum: threads add at most C terms one after the other, C = max(64, V / 256 + 13);
  so lse is off by at most  D = u (|M| + 2 E(M - z) + C + 3 |lse| + 8) + 2^-22, the log-prob by D + 3 u |logp|.
  * a gradient entry's softmax part: D + u (|M| + 2 (M - z_v) + 12) + 2^-21 relative, with bf16 logits one
    rounding of the kept exponential more (2^-8); then one rounding of the entry to its type (2^-8 or u).
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


def _rows(T, V, dt, seed, pad=0, offset=0, std=3.0, lift=12.0):
    """[T, V] logits in a buffer that is `pad` elements wider and starts `offset` elements in; half of the targets
    get much of their row's mass."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    z = torch.randn(T, V, generator=g, device=DEV) * std
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    up = lift * torch.rand(T, 1, generator=g, device=DEV) * (torch.arange(T, device=DEV)[:, None] % 2)
    z.scatter_add_(1, ids.long()[:, None], up)
    mask = (torch.rand(T, generator=g, device=DEV) < 0.7).to(torch.uint8)
    mask[T // 2] = 1
    buf = torch.full((T * (V + pad) + offset + 8,), 5.0, dtype=dt, device=DEV)
    view = buf[offset:offset + T * (V + pad)].view(T, V + pad)[:, :V]
    view.copy_(z.to(dt))
    return view, ids, mask, buf


def check(out, z, ids, mask, eps=0.0, zc=0.0, denom=None, rows=None):
    """Compare every output with the definition (of the rows listed, or all)."""
    logp, lse, loss, grad = out
    z64 = z.double().cpu().numpy()
    T, V = z64.shape
    r = o64.cross_entropy(z64, ids.cpu().numpy(), None if mask is None else mask.cpu().numpy(), eps, zc, denom)
    live = r["live"]
    lp = logp.double().cpu().numpy()
    assert np.array_equal(np.isnan(lp), ~live)
    C = max(64, V // 256 + 13)
    D = np.zeros(T)
    for t in np.flatnonzero(live):
        M = z64[t].max()
        e = np.exp(z64[t] - M)
        p = e / e.sum()
        below = np.where(p > 0, M - z64[t], 0.0)           # distances from the maximum, where they matter
        D[t] = U * (abs(M) + 2 * (p * below).sum() + C + 3 * abs(r["lse"][t]) + 8) + 2.0 ** -22
        if lse is not None:
            assert abs(lse[t].item() - r["lse"][t]) <= D[t], (t, lse[t].item(), r["lse"][t], D[t])
        assert abs(lp[t] - r["logp"][t]) <= D[t] + 3 * U * abs(r["logp"][t]), (t, lp[t], r["logp"][t], D[t])
        if grad is None:
            continue
        g = grad[t].double().cpu().numpy()
        bf = grad.dtype == BF
        half = 2.0 ** -8 if bf else U
        A = abs(1 + 2 * zc * r["lse"][t]) / r["n"]
        rel = D[t] + U * (abs(M) + 2 * below + 12) + 2.0 ** -21 + 2 * zc * D[t]
        part = A * p
        want = r["grad"][t]
        bound = part * (rel + (1.01 * 2.0 ** -8 if bf else 0.0)) + 1.01 * half * np.abs(want) + 8 * U * eps / V / r["n"]
        y = int(ids[t])
        others = 1.0 - p[y] if p[y] < 0.5 else np.delete(p, y).sum()
        bound[y] = ((others + 2 * zc * abs(r["lse"][t]) * p[y]) * (rel[y] + D[t]) / r["n"] + 1.01 * half * abs(want[y])
                    + 8 * U * (eps + 2 * zc * abs(r["lse"][t])) / r["n"])
        err = np.abs(g - want)
        # entries below the smallest normal number may be flushed
        ok = (err <= bound) | ((np.abs(want) < 2.0 ** -125) & (np.abs(g) < 2.0 ** -125))
        assert ok.all(), (t, np.flatnonzero(~ok)[:5], err[~ok][:5], bound[~ok][:5], y)
    if grad is not None:
        dead = torch.from_numpy(~live).to(DEV)
        assert not grad[dead].any()
    # the loss terms' errors add up; the sums themselves are fp64
    nll_tol = (D + 4 * U * np.nan_to_num(np.abs(r["logp"])))[live].sum() / r["n"]
    lse2_tol = ((2 * np.abs(r["lse"]) + 1) * (D + U * np.abs(r["lse"])))[live].sum() / r["n"]
    # the mean logit: C additions of terms z / V, and the differences around it
    mean_tol = sum(D[t] + (C + 8) * U * (np.abs(z64[t]).mean() + abs(z64[t].max())) for t in np.flatnonzero(live)) / r["n"] if eps else 0.0
    tol = [nll_tol + eps * mean_tol + zc * lse2_tol, nll_tol, mean_tol, lse2_tol]
    for k in range(4):
        assert abs(loss[k].item() - r["loss"][k]) <= tol[k] + 1e-12 * abs(r["loss"][k]), (k, loss[k].item(), r["loss"][k], tol[k])
    return r


def run(z, ids, mask, eps=0.0, zc=0.0, status=0, **kw):
    b = gc.binding()
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=eps, z_coef=zc, dev_status=st, **kw)
    assert st.item() == status, st.item()
    return out


SIZES = [(1, 1), (2, 2), (5, 7), (64, 1024), (33, 1000), (600, 264), (17, 4099), (12, 8192), (30, 32003), (8, 50304),
         (6, 50257), (5, 128256), (4, 151936), (3, 200000), (2, 262144), (2, 400003)]


@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("dt", [BF, F32])
def test_sizes_types_and_strides(T, V, dt):
    for k, (pad, offset) in enumerate([(0, 0), (8, 0), (3, 1), (5, 7)]):
        z, ids, mask, buf = _rows(T, V, dt, 7 * T + V + k, pad, offset)
        keep = buf.clone()
        check(run(z, ids, mask), z, ids, mask)
        check(run(z, ids, mask, 0.1, 1e-3), z, ids, mask, 0.1, 1e-3)
        assert torch.equal(buf, keep)                    # logits and what lies between the rows are only read
        # in place: the gradient replaces the rows and nothing between them
        a = run(z, ids, mask, 0.05, 0.0)
        b = run(z, ids, mask, 0.05, 0.0, in_place=True)
        assert b[3].data_ptr() == z.data_ptr() and torch.equal(a[3], b[3]) and torch.equal(a[2], b[2])
        z.fill_(5.0)
        assert (buf == 5.0).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_gradient_buffer_of_another_alignment_and_guard(dt):
    T, V = 9, 4099
    z, ids, mask, _ = _rows(T, V, dt, 1, pad=2, offset=0)
    ref = run(z, ids, mask, 0.1)
    for off in (0, 1, 3, 8):
        gbuf = torch.full((T * (V + 2) + 16,), 3.0, dtype=dt, device=DEV)
        g = gbuf[off:off + T * (V + 2)].view(T, V + 2)[:, :V]
        out = run(z, ids, mask, 0.1, grad_logits=g)
        check(out, z, ids, mask, 0.1)
        # an entry is c p - u, u = c eps / V: at most one rounding (2^-8) of c p and one of the entry in either call, so
        # the two are at most 2^-8 (|c p| + 2 |entry|) apart, |c p| <= |entry| + u, besides fp32 errors
        err = (g.double() - ref[3].double()).abs()
        u = 0.1 / V / max(int((mask != 0).sum()), 1)
        assert (err <= 1.05 * 2.0 ** -8 * (3 * ref[3].double().abs() + u)).all()
        g.fill_(3.0)
        assert (gbuf == 3.0).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [1000, 4099, 40000])
def test_infinities_lowest_values_and_nan(dt, V):
    low = torch.finfo(dt).min
    z, ids, mask, _ = _rows(12, V, dt, 3)
    mask.fill_(1)
    z[0, : V // 2] = float("-inf")               # a vocabulary cut in half
    ids[0] = V - 1
    z[1, 1:] = low                               # all the mass on one column
    ids[1] = 0
    z[2, 5:] = low
    ids[2] = 3
    z[3] = 1e30                                  # equal and huge
    z[4] = -1e30
    z[5, ids[5].long()] = 120.0                  # p_y rounds to one
    out = run(z, ids, mask)
    r = check(out, z, ids, mask)
    assert r["live"].all()
    assert (out[0][3:5] + np.log(V)).abs().max().item() <= 2.0 ** -20 * np.log(V)      # -log V, however large the logits
    z[6, V // 3] = float("nan")
    z[7] = float("-inf")
    z[8, 2] = float("inf")
    ids[9] = 1
    z[9, 1] = float("-inf")                      # the target itself impossible
    b = gc.binding()
    r = check(run(z, ids, mask, status=b.DEV_NONFINITE), z, ids, mask)
    assert r["live"].tolist() == [True] * 6 + [False] * 4 + [True] * 2
    # smoothing takes the mean logit: -inf anywhere takes the row out, the others are unchanged
    check(run(z, ids, mask, 0.1, status=b.DEV_NONFINITE), z, ids, mask, 0.1)
    # the same rows without loss weight are not looked at
    mask[6:10] = 0
    check(run(z, ids, mask), z, ids, mask)


@pytest.mark.parametrize("dt", [BF, F32])
def _check_live(out, z, ids, mask, eps=0.0, zc=0.0):
    """check() of a forward-only call, of the rows with a mask and a few others."""
    sel = mask != 0
    sel[::97] = True
    sub = tuple(None if t is None else t[sel] for t in out[:2])
    return check(sub + (out[2], None), z[sel], ids[sel], mask[sel], eps, zc)


@pytest.mark.parametrize("T,V", [(511, 20488), (512, 10241), (700, 10248), (600, 20480), (512, 20481), (513, 20487), (530, 32003),
                                 (512, 50304), (520, 151936), (3, 700001)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_forward_only_of_long_rows(T, V, dt):
    """Without a gradient a long row is cut into chunks that nobody joins before the second kernel."""
    b = gc.binding()
    for k, (pad, offset) in enumerate([(0, 0), (8, 0), (3, 1)]):
        z, ids, mask, buf = _rows(T, V, dt, 3 * T + V + k, pad, offset)
        mask[torch.arange(T, device=DEV) % 29 != 2] = 0
        mask[2 % T] = mask[T - 1] = 1
        keep = buf.clone()
        for eps, zc in ((0.0, 0.0), (0.1, 1e-3)):
            out = run(z, ids, mask, eps, zc, want_grad=False)
            _check_live(out, z, ids, mask, eps, zc)
        every = run(z, ids, None, 0.1, 1e-3, want_grad=False)
        assert torch.equal(every[0][mask != 0], out[0][mask != 0]) and torch.isfinite(every[0]).all()
        assert torch.isnan(run(z, ids, torch.zeros_like(mask), want_grad=False)[0]).all()
        assert torch.equal(buf, keep)
    if T < 100:
        return
    # rows that hold infinities, the lowest value, a NaN
    low = torch.finfo(dt).min
    mask[:8] = 1
    z[0, : V - 3] = float("-inf")
    ids[0] = V - 1
    z[1, 1:] = low
    ids[1] = 0
    z[2] = -1e30
    _check_live(run(z, ids, mask, want_grad=False), z, ids, mask)
    z[3, V // 3] = float("nan")
    z[4] = float("-inf")
    z[4, 7] = float("nan")
    z[5, V - 1] = float("inf")
    for eps in (0.0, 0.1):
        _check_live(run(z, ids, mask, eps, status=b.DEV_NONFINITE, want_grad=False), z, ids, mask, eps)
    ids[6] = V
    _check_live(run(z, ids, mask, status=b.DEV_NONFINITE | b.DEV_BAD_TARGET, want_grad=False), z, ids, mask)
    mask[3:7] = 0
    _check_live(run(z, ids, mask, want_grad=False), z, ids, mask)


def test_forward_only_captured_and_replayed():
    z, ids, mask, _ = _rows(600, 32003, BF, 17)
    eager = run(z, ids, mask, 0.1, want_grad=False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = gc.binding()
    with torch.cuda.stream(s):
        b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=0.1, want_grad=False)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=0.1, want_grad=False)
    mask0 = mask.clone()
    mask.copy_(1 - mask0)
    g.replay()
    flipped = [t.clone() for t in out[:3]]
    want = run(z, ids, mask, 0.1, want_grad=False)
    assert all(torch.equal(p.nan_to_num(9.0), q.nan_to_num(9.0)) for p, q in zip(flipped, want))
    mask.copy_(mask0)
    g.replay()
    assert all(torch.equal(p.nan_to_num(9.0), q.nan_to_num(9.0)) for p, q in zip(out[:3], eager))


def test_targets_out_of_range_and_ignored_ids():
    b = gc.binding()
    z, ids, mask, _ = _rows(20, 1000, BF, 5)
    mask.fill_(1)
    mask[:6] = 0
    ids[:6] = -100                               # a row without loss weight may carry any id
    check(run(z, ids, mask), z, ids, mask)
    ids[7], ids[8] = 1000, -1
    r = check(run(z, ids, mask, status=b.DEV_BAD_TARGET), z, ids, mask)
    assert r["n"] == 14 and not r["live"][7:9].any()


def test_masks_that_leave_nothing_or_everything():
    z, ids, mask, _ = _rows(40, 3000, BF, 6)
    nothing = torch.zeros_like(mask)
    logp, lse, loss, grad = run(z, ids, nothing, 0.1, 1e-4)
    assert torch.isnan(logp).all() and torch.isnan(lse).all() and not loss.any() and not grad.any()
    check(run(z, ids, None), z, ids, None)
    for v in (1, 2, 255):                         # any non-zero byte counts
        m = torch.where(mask != 0, torch.full_like(mask, v), mask)
        check(run(z, ids, m), z, ids, m)
    odd = torch.zeros(64, dtype=torch.uint8, device=DEV)[3:43]
    odd.copy_(mask)
    check(run(z, ids, odd), z, ids, odd)          # a mask that starts on no boundary


def test_outputs_asked_for_and_no_rows():
    b = gc.binding()
    z, ids, mask, _ = _rows(11, 2056, BF, 8)
    full = run(z, ids, mask, 0.1, 1e-3)
    fwd = run(z, ids, mask, 0.1, 1e-3, want_grad=False, want_lse=False)
    assert fwd[1] is None and fwd[3] is None and torch.equal(fwd[2], full[2])
    assert torch.equal(fwd[0].nan_to_num(9.0), full[0].nan_to_num(9.0))
    e = torch.empty((0, 2056), dtype=BF, device=DEV)
    logp, lse, loss, grad = run(e, ids[:0], mask[:0])
    assert logp.shape == (0,) and not loss.any() and grad.shape == (0, 2056)
    with pytest.raises(ValueError):
        b.rlf_cross_entropy_fwd_bwd(z, ids[:5], mask)
    with pytest.raises(ValueError):
        b.rlf_cross_entropy_fwd_bwd(z.t(), ids, mask)
    with pytest.raises(b.RlfError):
        b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=1.5)


def test_micro_batches_against_a_common_count_add_up():
    z, ids, mask, _ = _rows(30, 1500, F32, 9)
    n = (mask != 0).sum().reshape(1)
    whole = run(z, ids, mask, 0.1, 1e-3)
    parts = [run(z[a:b], ids[a:b], mask[a:b], 0.1, 1e-3, denom=n) for a, b in ((0, 1), (1, 17), (17, 30))]
    assert torch.equal(torch.cat([q[3] for q in parts]), whole[3])
    assert torch.allclose(sum(q[2] for q in parts), whole[2], rtol=1e-13, atol=0)


def test_gradient_against_differences():
    """Central differences of the call's own fp64 loss (fp32 logits, step 2^-5): truncation h^2 / 6 times a third
    derivative of at most one per row weight 1 / N, rounding of the loss terms (2^-22) over h."""
    z, ids, mask, _ = _rows(6, 40, F32, 10, std=1.0, lift=1.0)
    mask.fill_(1)
    eps, zc, h = 0.1, 1e-2, 2.0 ** -5
    grad = run(z, ids, mask, eps, zc)[3].clone()
    tol = (h * h / 6 * 1.5 + 4 * 2.0 ** -22 / h) / 6
    for t, v in ((0, 0), (1, int(ids[1])), (5, 39)):
        d = torch.zeros_like(z)
        d[t, v] = h
        fd = (run(z + d, ids, mask, eps, zc)[2][0] - run(z - d, ids, mask, eps, zc)[2][0]).item() / (2 * h)
        assert abs(fd - grad[t, v].item()) <= tol, (fd, grad[t, v].item())


@pytest.mark.parametrize("dt,V", [(BF, 32003), (BF, 151936), (F32, 1024)])
def test_repeated_captured_and_concurrent_calls(dt, V):
    T = 50
    z, ids, mask, _ = _rows(T, V, dt, 12)
    ref = run(z, ids, mask, 0.1, 1e-4)
    same = lambda o: all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(o, ref))
    for _ in range(5):
        assert same(run(z, ids, mask, 0.1, 1e-4))
    b = gc.binding()
    call = lambda: b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=0.1, z_coef=1e-4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    z0, ids0, mask0 = z.clone(), ids.clone(), mask.clone()
    z.copy_(z0.flip(0)), ids.copy_(ids0.flip(0)), mask.copy_(mask0.flip(0))
    g.replay()
    torch.cuda.synchronize()
    # (not the first result's rows in reverse: where a row's vectors begin decides which thread adds what)
    assert all(torch.equal(a.nan_to_num(7.0), b_.nan_to_num(7.0)) for a, b_ in zip(out, call()))
    check(out, z, ids, mask, 0.1, 1e-4)
    z.copy_(z0), ids.copy_(ids0), mask.copy_(mask0)
    g.replay()
    torch.cuda.synchronize()
    assert same(out)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(4):
        for st in streams:
            with torch.cuda.stream(st):
                outs.append(call())
    torch.cuda.synchronize()
    assert all(same(o) for o in outs)


def test_rows_past_32_bit_offsets():
    V, T = 151936, 14200                          # 2.16e9 logits
    z = torch.empty((T, V), dtype=BF, device=DEV)
    z.normal_(0, 3, generator=torch.Generator(device=DEV).manual_seed(1))
    ids = torch.randint(0, V, (T,), device=DEV, dtype=torch.int32)
    mask = (torch.arange(T, device=DEV) % 3 != 0).to(torch.uint8)
    n = (mask != 0).sum().reshape(1)
    out = run(z, ids, mask)
    tail = run(z[-40:].clone(), ids[-40:], mask[-40:], denom=n)
    assert torch.equal(out[3][-40:], tail[3]) and torch.equal(out[0][-40:].nan_to_num(1.0), tail[0].nan_to_num(1.0))
    last = slice(T - 3, T)
    check((out[0][last], out[1][last], run(z[last], ids[last], mask[last], denom=n)[2], out[3][last]), z[last], ids[last],
          mask[last], denom=int(n))


def test_agrees_with_the_log_prob_pass_and_the_grpo_gradient():
    """With advantage 1 and old = new the clipped-ratio surrogate's gradient is the cross entropy's: the two
    calls agree to their roundings."""
    b = gc.binding()
    z, ids, mask, _ = _rows(64, 50304, BF, 14)
    logp, _, _, grad = run(z, ids, mask)
    lp, _ = b.rlf_logp_entropy_fwd(z, ids)
    live = mask != 0
    assert (logp[live] - lp[live]).abs().max().item() <= 4e-5
    seq = torch.zeros(64, dtype=torch.int32, device=DEV)
    _, _, g2 = b.rlf_grpo_logp_loss_fwd_bwd(z, ids, seq, torch.ones(1, device=DEV), lp, lp, mask, 0.2, 0.0)
    err = (grad.double() - g2.double()).abs()
    assert (err <= 2.0 ** -5 * g2.double().abs() + 1e-12).all()
