"""The operators around a transformer block in plain fp64 numpy, written from their definitions: a linear layer
with its epilogue, and the norms after a block and before the next with the block's gate and residual scale.

TEST INFRASTRUCTURE ONLY: it shares no code with the CUDA package, which never imports it.
Arrays come in as fp64 (bf16 / fp32 inputs widened exactly by the caller).
"""
import math

import numpy as np

NONE, RELU, SILU, GELU, GELU_TANH = 0, 1, 2, 3, 4
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _logistic(u):
    u = np.asarray(u, np.float64)
    e = np.exp(-np.abs(u))
    return np.where(u >= 0, 1.0, e) / (1.0 + e)


def act(z, kind):
    if kind == RELU:
        return np.where(z < 0, 0.0, z)
    if kind == SILU:
        return z * _logistic(z)
    if kind == GELU:
        return z * 0.5 * _erfc(-z / math.sqrt(2.0))
    if kind == GELU_TANH:
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_grad(z, kind):
    if kind == RELU:
        return (z > 0).astype(np.float64)
    if kind == SILU:
        s = _logistic(z)
        return s + z * s * (1.0 - s)
    if kind == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == GELU_TANH:
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    return np.ones_like(z)


def linear(x, W, bias=None, kind=NONE, gated=False, residual=None):
    """-> (y, z)"""
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    n = z.shape[1] // 2
    y = act(z[:, :n], kind) * z[:, n:] if gated else act(z, kind)
    if residual is not None:
        y = y + np.asarray(residual, np.float64)
    return y, z


def linear_grad(dy, x, W, z=None, kind=NONE, gated=False):
    """-> (grad_x, grad_W, grad_bias, gz)"""
    dy, x, W = (np.asarray(a, np.float64) for a in (dy, x, W))
    if gated:
        n = dy.shape[1]
        gz = np.concatenate([dy * z[:, n:] * act_grad(z[:, :n], kind), dy * act(z[:, :n], kind)], axis=1)
    else:
        gz = dy if kind == NONE else dy * act_grad(z, kind)
    return gz @ W, gz.T @ x, gz.sum(axis=0), gz


def _unit(v, kind, eps):
    """kind: None (no norm), "rms" or "layer".  -> (normed rows before the weight, mean, 1 / spread)"""
    T = v.shape[0]
    if kind is None:
        return v, np.zeros(T), np.ones(T)
    mu = v.mean(axis=1) if kind == "layer" else np.zeros(T)
    c = v - mu[:, None]
    r = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
    return c * r[:, None], mu, r


def _gate(gate, form, beta):
    """form: None, "column" ([D]) or "row" ([T])"""
    if form is None:
        return np.full((1, 1), float(beta))
    g = beta * np.asarray(gate, np.float64)
    return g[None, :] if form == "column" else g[:, None]


def block_norm(x, residual, post=None, post_w=None, post_b=None, pre=None, pre_w=None, pre_b=None, gate=None, form=None,
               alpha=1.0, beta=1.0, eps=1e-6):
    """h = alpha residual + beta gate norm_post(x);  y = norm_pre(h).  -> (h, y | None, stats [4, T])"""
    x, residual = np.asarray(x, np.float64), np.asarray(residual, np.float64)
    n, m1, r1 = _unit(x, post, eps)
    if post is not None:
        n = n * post_w + (0.0 if post_b is None else post_b)
    h = alpha * residual + _gate(gate, form, beta) * n
    u, m2, r2 = _unit(h, pre, eps)
    y = None if pre is None else u * pre_w + (0.0 if pre_b is None else pre_b)
    return h, y, np.stack([m1, r1, m2, r2])


def block_norm_grad(dy, dh, x, h, stats, post=None, post_w=None, post_b=None, pre=None, pre_w=None, gate=None, form=None,
                    alpha=1.0, beta=1.0):
    """-> dict(x, residual, gate, post_weight, post_bias, pre_weight, pre_bias), the gradients that exist"""
    x, h = np.asarray(x, np.float64), np.asarray(h, np.float64)
    m1, r1, m2, r2 = (np.asarray(s, np.float64)[:, None] for s in stats)
    gh = np.zeros_like(x) if dh is None else np.array(dh, np.float64)
    out = {}

    def through(g, w, u, r, kind):
        q = g * w
        d = q - u * (q * u).mean(axis=1, keepdims=True)
        if kind == "layer":
            d = d - q.mean(axis=1, keepdims=True)
        return d * r

    if pre is not None:
        dy = np.asarray(dy, np.float64)
        u = (h - m2) * r2
        gh = gh + through(dy, pre_w, u, r2, pre)
        out["pre_weight"], out["pre_bias"] = (dy * u).sum(axis=0), dy.sum(axis=0)
    out["residual"] = alpha * gh
    gn = _gate(gate, form, beta) * gh
    n = x
    if post is not None:
        u = (x - m1) * r1
        out["x"] = through(gn, post_w, u, r1, post)
        out["post_weight"], out["post_bias"] = (gn * u).sum(axis=0), gn.sum(axis=0)
        n = u * post_w + (0.0 if post_b is None else post_b)
    else:
        out["x"] = gn
    if form is not None:
        out["gate"] = (beta * gh * n).sum(axis=0 if form == "column" else 1)
    return out
