"""GPU parity of rlf_cross_entropy_fwd_bwd where a cluster of CTAs takes many rows one after the other.

The bounds are those that tests/test_gpu_cross_entropy.py derives, evaluated for all rows at once in 64 bits on the GPU.
"""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def rows(T, V, dt, seed, pad=0, offset=0, live=0.5, std=3.0, lift=12.0):
    """[T, V] logits in a buffer `pad` elements wider that starts `offset` elements in, targets, loss mask, the buffer."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.full((T * (V + pad) + offset + 8,), 5.0, dtype=dt, device=DEV)
    z = buf[offset:offset + T * (V + pad)].view(T, V + pad)[:, :V]
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    for a in range(0, T, 4096):
        b = min(T, a + 4096)
        x = torch.randn(b - a, V, generator=g, device=DEV) * std
        up = lift * torch.rand(b - a, 1, generator=g, device=DEV) * (torch.arange(b - a, device=DEV)[:, None] % 2)
        x.scatter_add_(1, ids[a:b].long()[:, None], up)
        z[a:b] = x.to(dt)
    mask = (torch.rand(T, generator=g, device=DEV) < live).to(torch.uint8)
    mask[T // 2] = 1
    return z, ids, mask, buf


def run(z, ids, mask, eps=0.0, zc=0.0, status=0, **kw):
    b = gc.binding()
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = b.rlf_cross_entropy_fwd_bwd(z, ids, mask, label_smoothing=eps, z_coef=zc, dev_status=st, **kw)
    assert st.item() == status, st.item()
    return out


def check(out, z, ids, mask, eps=0.0, zc=0.0):
    """Every row's log-prob, log-sum-exp and gradient; every row of finite logits is live where mask is set."""
    logp, lse, loss, grad = out
    T, V = z.shape
    live = mask != 0
    n = max(int(live.sum()), 1)
    assert torch.equal(torch.isnan(logp), ~live) and (lse is None or torch.equal(torch.isnan(lse), ~live))
    if grad is not None:
        assert not grad[~live].any()
    C = max(64, V // 256 + 13)
    bf = z.dtype == BF
    half = 2.0 ** -8 if bf else U
    at = torch.nonzero(live).flatten()
    step = max(1, (1 << 26) // V)
    nll = 0.0
    tol = 0.0
    for a in range(0, at.numel(), step):
        r = at[a:a + step]
        x = z[r].double()
        y = ids[r].long()[:, None]
        M = x.max(dim=1, keepdim=True).values
        l = torch.logsumexp(x, dim=1, keepdim=True)
        lp = torch.log_softmax(x, dim=1)
        p = lp.exp()
        below = torch.where(p > 0, M - x, torch.zeros_like(x))
        D = U * (M.abs() + 2 * (p * below).sum(dim=1, keepdim=True) + C + 3 * l.abs() + 8) + 2.0 ** -22
        want_lp = lp.gather(1, y)
        err = (logp[r].double()[:, None] - want_lp).abs()
        lim = D + 3 * U * want_lp.abs()
        assert (err <= lim).all(), ((err / lim).max().item(), r[(err / lim).argmax()].item())
        nll += -want_lp.sum().item()
        tol += (D + 4 * U * want_lp.abs()).sum().item()
        if lse is not None:
            assert ((lse[r].double()[:, None] - l).abs() <= D).all()
        if grad is None:
            continue
        A = (1 + 2 * zc * l).abs() / n
        want = (1 + 2 * zc * l) * p - eps / V
        others = torch.where(torch.arange(V, device=DEV) == y, torch.zeros_like(p), p).sum(dim=1, keepdim=True)
        py = p.gather(1, y)
        want.scatter_(1, y, 2 * zc * l * py - others + eps - eps / V)
        want /= n
        rel = D + U * (M.abs() + 2 * below + 12) + 2.0 ** -21 + 2 * zc * D
        bound = A * p * (rel + (1.01 * 2.0 ** -8 if bf else 0.0)) + 1.01 * half * want.abs() + 8 * U * eps / V / n
        wy = want.gather(1, y).abs()
        bound.scatter_(1, y, (others + 2 * zc * l.abs() * py) * (rel.gather(1, y) + D) / n + 1.01 * half * wy
                       + 8 * U * (eps + 2 * zc * l.abs()) / n)
        g = grad[r].double()
        err = (g - want).abs()
        ok = (err <= bound) | ((want.abs() < 2.0 ** -125) & (g.abs() < 2.0 ** -125))
        assert ok.all(), (r[torch.nonzero(~ok)[0, 0]].item(), torch.nonzero(~ok)[:4].tolist(), (err / bound)[~ok][:4])
    assert abs(loss[1].item() - nll / n) <= tol / n + 1e-12 * abs(nll / n)


# The last vector of a row lies with thread 31 or 32 (63 or 64 with the longer rows), by where the row starts
@pytest.mark.parametrize("dt,V", [(BF, 252), (BF, 508), (F32, 126), (F32, 254)])
def test_edges_of_the_last_live_row_before_a_row_without_loss(dt, V):
    """Rows whose first and last vectors are stored by element: a cluster's last live row is followed by rows that are
    zeroed, whose last vector another warp may hold."""
    z, ids, mask, _ = rows(60000, V, dt, V, pad=1, offset=1)
    for live in (mask, torch.ones_like(mask)):
        for _ in range(3):
            check(run(z, ids, live), z, ids, live)


@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_shorter_than_a_vector_on_any_base(dt):
    """Several rows share the 16-byte vector that the logits start in; what lies before the base (and behind the rows) is
    neither part of a row nor written."""
    for V in (1, 2, 3, 7):
        for pad in (0, 1):
            for offset in range(0, 8):
                z, ids, mask, buf = rows(41, V, dt, V + offset, pad, offset)
                buf[:offset] = float("nan")
                keep = buf.clone()
                out = run(z, ids, mask, 0.1)
                check(out, z, ids, mask, 0.1)
                assert torch.equal(buf[offset:], keep[offset:])
                same = run(z, ids, mask, 0.1, in_place=True)
                assert torch.equal(same[3], out[3])
                z.fill_(5.0)
                assert torch.isnan(buf[:offset]).all() and (buf[offset:] == 5.0).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T", [8, 600])
def test_nan_that_a_warp_sees_with_no_finite_logit(dt, T):
    """A NaN whose neighbours in the same warp are -inf, the target, or nothing at all still takes its row out: NaN
    statistics, a zero gradient, the status; with a gradient or without one, on the cluster and the chunked kernels."""
    b = gc.binding()
    nan, inf = float("nan"), float("inf")
    vec = 8 if dt == BF else 4
    for V in (32 * vec, 32 * vec + 1, 33 * vec, 1000, 2048 * vec + 8, 2600 * vec + 1):
        z, ids, mask, _ = rows(T, V, dt, V, live=1.1)
        ids[:6] = V // 2
        z[0, V - 1] = nan                       # the last column, perhaps its warp's only one
        z[1] = nan
        z[1, V // 2] = 1.0                      # nothing but the target is a number
        z[2] = -inf
        z[2, V // 2], z[2, V - 1] = 0.5, nan    # a masked vocabulary with one NaN
        z[3] = -inf
        z[3, V // 2], z[3, 0] = 0.5, 0.25       # a masked vocabulary, sound
        z[4] = nan
        z[5, :V // 2] = nan
        dead = torch.tensor([0, 1, 2, 4, 5], device=DEV)
        sound = torch.ones_like(mask)
        sound[dead] = 0
        for eps in (0.0, 0.1):
            gone = sound.clone()
            if eps:
                gone[3] = 0                     # (the mean logit of -inf)
            for grad in (True, False):
                lp, lse, loss, g = run(z, ids, mask, eps, status=b.DEV_NONFINITE, want_grad=grad)
                assert torch.equal(torch.isnan(lp), gone == 0) and torch.equal(torch.isnan(lse), gone == 0), (V, eps, grad)
                assert torch.isfinite(loss).all()
                if grad:
                    assert torch.isfinite(g).all() and not g[gone == 0].any()
            # the others are what they are without the bad rows (their count apart)
            n = torch.full((1,), T, dtype=torch.int64, device=DEV)
            a, c = run(z, ids, mask, eps, status=b.DEV_NONFINITE, denom=n), run(z, ids, gone, eps, denom=n)
            assert torch.equal(a[0].nan_to_num(7.0), c[0].nan_to_num(7.0)) and torch.equal(a[2], c[2]) and torch.equal(a[3], c[3])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,V,grad", [(768, 1024, True), (768, 20488, True), (768, 20488, False), (768, 5003, True)])
def test_log_prob_of_rows_far_from_zero(dt, T, V, grad):
    """Rows around +-40 ... 4000.  The differences z - max are exact there, so the log-prob keeps the digits that it has
    around zero: an exponential 2^-22 and u (2 (M - z)) relative, the sum C additions, the logarithm and the last difference
    u each (u = 2^-24, C as in check()); a maximum M itself leaves no error.  The log-sum-exp has u |M| from its rounding."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    z = (2.0 * torch.randn(T, V, generator=g, device=DEV)).to(BF).float()
    z -= z.max(dim=1, keepdim=True).values
    far = torch.exp(torch.rand(T, 1, generator=g, device=DEV) * 4.6 + 3.7) * (1 - 2 * (torch.arange(T, device=DEV)[:, None] % 2))
    z = (z + far.to(BF).float()).to(dt)
    ids = z.argmax(dim=1).int()
    other = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    ids = torch.where(torch.arange(T, device=DEV) % 3 == 0, other, ids)
    logp, lse, loss, gr = run(z, ids, None, want_grad=grad)
    x = z.double()
    M = x.max(dim=1, keepdim=True).values
    want = torch.log_softmax(x, dim=1)
    p = want.exp()
    below = torch.where(p > 0, M - x, torch.zeros_like(x))
    C = max(64, V // 256 + 13)
    lp = want.gather(1, ids.long()[:, None])[:, 0]
    D = U * (2 * (p * below).sum(dim=1) + C + 8) + 2.0 ** -22 + 3 * U * lp.abs()
    err = (logp.double() - lp).abs()
    assert (err <= D).all(), ((err / D).max().item(), err.max().item())
    assert ((lse.double() - torch.logsumexp(x, dim=1)).abs() <= D + U * M[:, 0].abs() * 2).all()
    if grad and dt == BF:
        # two roundings to bf16 (the kept exponential and the entry), and the errors above
        want_g = p / T
        want_g.scatter_add_(1, ids.long()[:, None], torch.full((T, 1), -1.0 / T, dtype=torch.float64, device=DEV))
        rel = D[:, None] + U * (2 * below + 12) + 2.0 ** -21 + 2.02 * 2.0 ** -8
        off = torch.ones_like(p, dtype=torch.bool).scatter_(1, ids.long()[:, None], False)
        e = (gr.double() - want_g).abs()
        assert (e <= rel * p / T + 2.0 ** -125)[off].all()


# by launch shape: CTAs of 64 and 128 threads, clusters of 1, 2, 4, 8, 10 and 16 CTAs; several rows per cluster each
@pytest.mark.parametrize("T,V", [(15000, 504), (7000, 6007), (6500, 8000), (3200, 16001), (1700, 30016), (1600, 32003), (800, 70001),
                                 (450, 151936), (420, 151937), (260, 196001), (160, 300008), (90, 500001)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_many_rows_per_cluster(dt, T, V):
    if dt == F32:
        V = (V + 1) // 2
    for pad, offset in ((0, 0), (3, 1)):
        z, ids, mask, buf = rows(T, V, dt, T + V + pad, pad, offset, live=0.7)
        for eps, zc in ((0.0, 0.0), (0.1, 1e-3)):
            out = run(z, ids, mask, eps, zc)
            check(out, z, ids, mask, eps, zc)
            again = run(z, ids, mask, eps, zc)
            assert torch.equal(again[3], out[3]) and torch.equal(again[2], out[2])
        same = run(z, ids, mask, 0.1, 1e-3, in_place=True)
        assert torch.equal(same[3], out[3])
        z.fill_(5.0)
        assert (buf == 5.0).all()
