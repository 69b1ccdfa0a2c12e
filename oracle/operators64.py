"""The supervised-stage operators in plain fp64 numpy, written from their definitions.

TEST INFRASTRUCTURE ONLY: it shares no code with the CUDA package, which never imports it.
Arrays come in as fp64 (bf16 / fp32 inputs widened exactly by the caller).
"""
import numpy as np


def cross_entropy(z, ids, mask=None, smoothing=0.0, z_coef=0.0, denom=None):
    """z [T, V].  A row takes part where mask != 0, its target lies in the vocabulary and its log-sum-exp and
    loss term are finite; the denominator counts the mask as given.
    -> dict(logp, lse [T] (NaN where a row does not take part), loss [4], grad [T, V], coef [T], live [T])"""
    z = np.asarray(z, np.float64)
    T, V = z.shape
    ids = np.asarray(ids, np.int64)
    m = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    n = max(int(m.sum()) if denom is None else int(denom), 1)
    logp, lse = np.full(T, np.nan), np.full(T, np.nan)
    grad = np.zeros((T, V))
    loss = np.zeros(4)
    live = np.zeros(T, bool)
    for t in range(T):
        y = ids[t]
        if not m[t] or y < 0 or y >= V:
            continue
        row = z[t]
        with np.errstate(all="ignore"):
            top = row.max()
            s = np.exp(row - top).sum()
            l = top + np.log(s)
            lp = (row[y] - top) - np.log(s)
            smooth = l - (row / V).sum() if smoothing else 0.0
        if not (np.isfinite(l) and np.isfinite(lp) and np.isfinite(smooth)):
            continue
        live[t] = True
        logp[t], lse[t] = lp, l
        loss += np.array([(1 - smoothing) * -lp + smoothing * smooth + z_coef * l * l, -lp, smooth, l * l])
        p = np.exp(row - top) / s
        g = (1 + 2 * z_coef * l) * p - smoothing / V
        # p_y - (1 - smoothing) with 1 - p_y summed over the other columns: no cancellation as p_y -> 1
        others = np.delete(np.exp(row - top), y).sum() / s
        g[y] = smoothing - others + 2 * z_coef * l * p[y] - smoothing / V
        grad[t] = g / n
    return dict(logp=logp, lse=lse, loss=loss / n, grad=grad, live=live, n=n)


def fused_cross_entropy(H, W, ids, mask=None, smoothing=0.0, z_coef=0.0, denom=None):
    """The same with z = H W^T.  -> the dict of cross_entropy plus grad_hidden [T, D], grad_W [V, D]"""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    with np.errstate(invalid="ignore"):
        r = cross_entropy(H @ W.T, ids, mask, smoothing, z_coef, denom)
    r["grad_hidden"] = r["grad"] @ W
    on = r["live"]                      # a row that does not take part may hold anything
    r["grad_W"] = r["grad"][on].T @ H[on]
    return r


def norm(x, weight, bias=None, residual=None, layer=False, eps=1e-6):
    """-> (y, h, mean, rstd)"""
    h = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    mu = h.mean(axis=1) if layer else np.zeros(h.shape[0])
    c = h - mu[:, None]
    r = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
    y = c * r[:, None] * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, h, mu, r


def norm_grad(dy, x, weight, mean, rstd, layer=False, skip=None):
    """-> (grad_x, grad_weight, grad_bias)"""
    dy, x, w = (np.asarray(a, np.float64) for a in (dy, x, weight))
    r = np.asarray(rstd, np.float64)[:, None]
    xh = (x - (np.asarray(mean, np.float64)[:, None] if layer else 0.0)) * r
    g = dy * w
    dx = g - xh * (g * xh).mean(axis=1, keepdims=True)
    if layer:
        dx = dx - g.mean(axis=1, keepdims=True)
    dx = dx * r
    if skip is not None:
        dx = dx + np.asarray(skip, np.float64)
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)
