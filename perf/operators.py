"""The supervised-stage operators of the policy head, as they are measured: softmax cross entropy over
the vocabulary (from logits, and fused with the LM head so that the logits are never kept), and the
final norm in front of the head, forward and backward.

`own = False` computes every operator in elementary torch operations in fp32; `own = True` makes the
library calls of paper_2509_06980_b200.binding.  Both take the same prepared inputs.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
RMS, LAYER = "rms", "layer"
DEV = "cuda"


# ---------------------------------------------------------------------------------------------
# cases
def _norm(op, T, D, dt=BF16, w_dt=BF16, kind=RMS, bias=False, residual=False, pad=0):
    return dict(op=op, T=T, D=D, dt=dt, w_dt=w_dt, kind=kind, bias=bias, residual=residual, pad=pad)


def _ce(T, V, dt=BF16, live=0.54, smoothing=0.0, z_coef=0.0, grad=True, pad=0):
    return dict(op="ce", T=T, V=V, dt=dt, live=live, smoothing=smoothing, z_coef=z_coef, grad=grad, pad=pad)


def _head(T, D, V, live=0.54, smoothing=0.0, z_coef=0.0, grad=True):
    return dict(op="head", T=T, D=D, V=V, live=live, smoothing=smoothing, z_coef=z_coef, grad=grad)


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # sampling a handful of responses token by token: one norm call per step, latency is all that counts
    add("norm_fwd_decode", _norm("norm_fwd", 8, 2560, residual=True))
    # the training micro-batch of the 4B-shaped recipe (16 responses of 2048 tokens), residual add folded in
    add("norm_fwd_microbatch", _norm("norm_fwd", 32768, 2560, residual=True))
    # a small fp32 reward model's layer norm with bias, a ragged batch and a width that fills no vector
    add("norm_fwd_layer_odd", _norm("norm_fwd", 4999, 1021, dt=F32, w_dt=F32, kind=LAYER, bias=True))
    # the backward of a short last micro-batch at the 8B-shaped width
    add("norm_bwd_short", _norm("norm_bwd", 65, 4096))
    # the training micro-batch again: gradient of the residual stream added in, weight gradient reduced over 32768 rows
    add("norm_bwd_microbatch", _norm("norm_bwd", 32768, 2560, residual=True))
    # layer norm with bias over one 8192-token response less its prompt, fp32 weights beside bf16 activations
    add("norm_bwd_layer", _norm("norm_bwd", 8191, 4096, w_dt=F32, kind=LAYER, bias=True))
    # the tiny fp32 recipe (16 responses of 64 tokens, V = 1024): launches count
    add("ce_tiny_f32", _ce(1024, 1024, dt=F32, live=0.7))
    # a vocabulary that fills no vector, rows of a wider buffer, label smoothing
    add("ce_odd_smoothed", _ce(4099, 32003, smoothing=0.1, pad=5))
    # one 8192-token response over the recipes' full vocabulary, with the z-loss that keeps lse near zero
    add("ce_full_vocabulary", _ce(8192, 151936, z_coef=1e-4))
    # a few tokens against the whole 4B-shaped head: reading the head and writing its gradient is the cost
    add("head_few_tokens", _head(64, 2560, 151936, live=0.8))
    # an ordinary fine-tuning micro-batch on a 32000-entry vocabulary, smoothing and z-loss on
    add("head_smoothed", _head(2047, 2048, 32000, live=0.7, smoothing=0.1, z_coef=1e-4))
    # the 8B-shaped recipe's micro-batch: 8192 tokens, D = 4096, the full vocabulary
    add("head_microbatch_8b", _head(8192, 4096, 151936))
    return c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "ce", "head"])
    if op in ("norm_fwd", "norm_bwd"):
        D = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            D = (D + 63) // 64 * 64
        T = _log_int(rng, 1, max(1, min(65536, 32768 * 2560 // D)))
        kind = rng.choice([RMS, LAYER])
        return _norm(op, T, D, dt=rng.choice([BF16, BF16, F32]), w_dt=rng.choice([BF16, F32]), kind=kind,
                     bias=kind == LAYER and rng.random() < 0.7, residual=rng.random() < 0.5,
                     pad=rng.choice([0, 0, 8, 3]))
    smoothing = rng.choice([0.0, 0.0, 0.05, 0.1])
    z_coef = rng.choice([0.0, 1e-4])
    live = round(rng.uniform(0.3, 1.0), 2)
    grad = rng.random() < 0.8
    if op == "ce":
        V = _log_int(rng, 512, 200000)
        if rng.random() < 0.6:
            V = (V + 7) // 8 * 8
        dt = rng.choice([BF16, BF16, F32])
        T = _log_int(rng, 1, max(1, 8192 * 151936 // (V * (2 if dt == F32 else 1))))
        T = min(T, 65536)
        return _ce(T, V, dt=dt, live=live, smoothing=smoothing, z_coef=z_coef, grad=grad, pad=rng.choice([0, 0, 8, 3]))
    D = (_log_int(rng, 64, 4096) + 63) // 64 * 64
    V = (_log_int(rng, 512, 151936) + 7) // 8 * 8
    T = _log_int(rng, 1, 8192)
    return _head(T, D, V, live=live, smoothing=smoothing, z_coef=z_coef, grad=grad)


# ---------------------------------------------------------------------------------------------
# inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(shape, g, dt=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dt)


def _spans(T, live, g):
    """Loss mask of multi-turn responses: runs of 32 tokens that are the model's own or tool output."""
    runs = torch.rand((T + 31) // 32, generator=g, device=DEV) < live
    mask = runs.repeat_interleave(32)[:T].contiguous()
    mask[T - 1] = True
    return mask.to(torch.uint8)


def _padded(rows, pad, g, dt, scale):
    """[T, D] rows of a buffer that is `pad` elements wider."""
    T, D = rows
    return _randn((T, D + pad), g, dt, scale)[:, :D]


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd"):
        T, D, dt, w_dt = case["T"], case["D"], _DT[case["dt"]], _DT[case["w_dt"]]
        st = dict(case=case, weight=(1.0 + 0.2 * _randn((D,), g)).to(w_dt),
                  bias=_randn((D,), g, w_dt, 0.1) if case["bias"] else None)
        # the residual stream: a few columns far larger than the others, a small offset
        x = _randn((T, D + case["pad"]), g, torch.float32, 2.0) + 0.25
        x[:, :: max(1, D // 7)] *= 8.0
        st["x"] = x.to(dt)[:, :D]
        if op == "norm_fwd":
            st["residual"] = _padded((T, D), case["pad"], g, dt, 1.0) if case["residual"] else None
        else:
            st["grad_y"] = _randn((T, D), g, dt, 1e-3)
            st["grad_skip"] = _randn((T, D), g, dt, 1e-3) if case["residual"] else None
            xf = st["x"].float()
            mean = xf.mean(dim=1) if case["kind"] == LAYER else None
            xc = xf if mean is None else xf - mean[:, None]
            st["mean"] = mean
            st["rstd"] = torch.rsqrt((xc * xc).mean(dim=1) + EPS)
        return st
    T, V = case["T"], case["V"]
    st = dict(case=case, mask=_spans(T, case["live"], g),
              ids=torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32))
    if op == "ce":
        z = torch.randn((T, V + case["pad"]), generator=g, device=DEV, dtype=torch.float32)
        z *= 3.0
        # a trained model puts much of its mass on many of the targets
        lift = 16.0 * torch.rand((T, 1), generator=g, device=DEV)
        z.scatter_add_(1, st["ids"].long()[:, None], lift)
        st["logits"] = z.to(_DT[case["dt"]])[:, :V]
    else:
        D = case["D"]
        st["hidden"] = _randn((T, D), g, torch.bfloat16)
        st["W"] = _randn((V, D), g, torch.bfloat16, 2.0 / math.sqrt(D))
    return st


EPS = 1e-6


# ---------------------------------------------------------------------------------------------
# plain forms (fp32, elementary operations)
def _norm_fwd_plain(s):
    case = s["case"]
    dt = s["x"].dtype
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    mean = h.mean(dim=1) if case["kind"] == LAYER else None
    hc = h if mean is None else h - mean[:, None]
    rstd = torch.rsqrt((hc * hc).mean(dim=1) + EPS)
    y = hc * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = dict(y=y.to(dt), rstd=rstd)
    if mean is not None:
        out["mean"] = mean
    if s["residual"] is not None:
        out["sum"] = h.to(dt)
    return out


def _norm_bwd_plain(s):
    case = s["case"]
    dt = s["x"].dtype
    dy, rstd = s["grad_y"].float(), s["rstd"][:, None]
    xh = s["x"].float()
    if s["mean"] is not None:
        xh = xh - s["mean"][:, None]
    xh = xh * rstd
    gr = dy * s["weight"].float()
    dx = gr - xh * (gr * xh).mean(dim=1, keepdim=True)
    if s["mean"] is not None:
        dx = dx - gr.mean(dim=1, keepdim=True)
    dx = dx * rstd
    if s["grad_skip"] is not None:
        dx = dx + s["grad_skip"].float()
    out = dict(grad_x=dx.to(dt), grad_weight=(dy * xh).sum(dim=0))
    if case["bias"]:
        out["grad_bias"] = dy.sum(dim=0)
    return out


def _ce_rows(z, s):
    """-> per-token log-prob and lse (NaN where the mask is 0), the four loss means (total, negative
    log-prob, smoothing term, lse^2; the third is 0 without smoothing), dL/dz or None."""
    case = s["case"]
    eps, zc, V = case["smoothing"], case["z_coef"], case["V"]
    live = s["mask"] != 0
    n = live.sum().clamp(min=1)
    y = s["ids"].long()[:, None]
    m = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - m)
    S = e.sum(dim=1, keepdim=True)
    lse = m + torch.log(S)
    logp = (z.gather(1, y) - m) - torch.log(S)
    smooth = lse - z.mean(dim=1, keepdim=True) if eps else torch.zeros_like(lse)
    nan = torch.full_like(lse, float("nan"))
    terms = torch.cat([(1.0 - eps) * -logp + eps * smooth + zc * lse * lse, -logp, smooth, lse * lse], dim=1)
    loss = torch.where(live[:, None], terms, torch.zeros_like(terms)).double().sum(dim=0) / n
    out = dict(logp=torch.where(live[:, None], logp, nan)[:, 0], lse=torch.where(live[:, None], lse, nan)[:, 0],
               loss=loss.float())
    if not case["grad"]:
        return out, None
    dz = e * ((1.0 + 2.0 * zc * lse) / S)
    if eps:
        dz -= eps / V
    dz.scatter_add_(1, y, torch.full_like(lse, -(1.0 - eps)))
    dz *= live[:, None].float() / n
    return out, dz


def _ce_plain(s):
    out, dz = _ce_rows(s["logits"].float(), s)
    if dz is not None:
        out["grad_logits"] = dz.to(s["logits"].dtype)
    return out


def _head_plain(s):
    H, W = s["hidden"].float(), s["W"].float()
    out, dz = _ce_rows(H @ W.t(), s)
    if dz is not None:
        out["grad_hidden"] = (dz @ W).to(torch.bfloat16)
        out["grad_W"] = (dz.t() @ H).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------------------------------------
# the library's calls
def _own(s):
    from paper_2509_06980_b200 import binding as rlf

    case = s["case"]
    op = case["op"]
    if op == "norm_fwd":
        y, total, mean, rstd = rlf.rlf_norm_fwd(s["x"], s["weight"], bias=s["bias"], residual=s["residual"],
                                                kind=rlf.NORM_LAYER if case["kind"] == LAYER else rlf.NORM_RMS, eps=EPS)
        out = dict(y=y, rstd=rstd)
        if mean is not None:
            out["mean"] = mean
        if total is not None:
            out["sum"] = total
        return out
    if op == "norm_bwd":
        gx, gw, gb = rlf.rlf_norm_bwd(s["grad_y"], s["x"], s["weight"], s["mean"], s["rstd"],
                                      kind=rlf.NORM_LAYER if case["kind"] == LAYER else rlf.NORM_RMS,
                                      grad_skip=s["grad_skip"], want_grad_bias=case["bias"])
        out = dict(grad_x=gx, grad_weight=gw)
        if gb is not None:
            out["grad_bias"] = gb
        return out
    if op == "ce":
        logp, lse, loss, grad = rlf.rlf_cross_entropy_fwd_bwd(s["logits"], s["ids"], s["mask"],
                                                              label_smoothing=case["smoothing"], z_coef=case["z_coef"],
                                                              want_grad=case["grad"])
        out = dict(logp=logp, lse=lse, loss=loss.float())
        if grad is not None:
            out["grad_logits"] = grad
        return out
    logp, lse, loss, gh, gw = rlf.rlf_fused_lmhead_cross_entropy(s["hidden"], s["W"], s["ids"], s["mask"],
                                                                 label_smoothing=case["smoothing"],
                                                                 z_coef=case["z_coef"], want_grad_hidden=case["grad"],
                                                                 want_grad_W=case["grad"], grad_W_dtype=torch.bfloat16)
    out = dict(logp=logp, lse=lse, loss=loss.float())
    if gh is not None:
        out["grad_hidden"], out["grad_W"] = gh, gw
    return out


_PLAIN = dict(norm_fwd=_norm_fwd_plain, norm_bwd=_norm_bwd_plain, ce=_ce_plain, head=_head_plain)


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
def work(case):
    op = case["op"]
    T = case["T"]
    if op in ("norm_fwd", "norm_bwd"):
        D, esz, wsz = case["D"], 2 if case["dt"] == BF16 else 4, 2 if case["w_dt"] == BF16 else 4
        stats = T * (8 if case["kind"] == LAYER else 4)
        if op == "norm_fwd":
            nbytes = T * D * esz * (4 if case["residual"] else 2) + D * wsz * (2 if case["bias"] else 1) + stats
            return dict(bytes=nbytes, flops=8 * T * D)
        nbytes = T * D * esz * (4 if case["residual"] else 3) + D * wsz + 4 * D * (2 if case["bias"] else 1) + stats
        return dict(bytes=nbytes, flops=14 * T * D)
    V = case["V"]
    n_live = case["live"] * T
    per_token = 13 * T
    if op == "ce":
        esz = 2 if case["dt"] == BF16 else 4
        return dict(bytes=V * esz * (n_live + (T if case["grad"] else 0)) + per_token, flops=6 * V * n_live)
    D = case["D"]
    nbytes = 2 * D * (n_live + V) + (2 * D * (T + V) if case["grad"] else 0) + per_token
    return dict(bytes=nbytes, flops=(6 if case["grad"] else 2) * n_live * V * D)


# ---------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm_fwd":
        h = s["x"].double()
        if s["residual"] is not None:
            h += s["residual"].double()
        layer = case["kind"] == LAYER
        mu = h.sum(dim=1) / case["D"]
        spread = ((h - mu[:, None]) ** 2 if layer else h ** 2).sum(dim=1) / case["D"]
        rstd = 1.0 / torch.sqrt(spread + EPS)
        y = ((h - mu[:, None]) if layer else h) * rstd[:, None] * s["weight"].double()[None, :]
        if s["bias"] is not None:
            y += s["bias"].double()[None, :]
        out = dict(y=y, rstd=rstd)
        if layer:
            out["mean"] = mu
        if s["residual"] is not None:
            out["sum"] = h
        return out
    if op == "norm_bwd":
        x, dy, r = s["x"].double(), s["grad_y"].double(), s["rstd"].double()
        layer = case["kind"] == LAYER
        mu = s["mean"].double() if layer else torch.zeros_like(r)
        D = case["D"]
        w = s["weight"].double()
        xh = (x - mu[:, None]) * r[:, None]
        a = torch.einsum("td,td,d->t", dy, xh, w) / D
        b = (dy @ w) / D if layer else torch.zeros_like(r)
        dx = (dy * w - b[:, None] - xh * a[:, None]) * r[:, None]
        if s["grad_skip"] is not None:
            dx += s["grad_skip"].double()
        out = dict(grad_x=dx, grad_weight=torch.einsum("td,td->d", dy, xh))
        if case["bias"]:
            out["grad_bias"] = dy.sum(dim=0)
        return out
    # cross entropy, a block of rows at a time; only live rows take part
    T, V, eps, zc = case["T"], case["V"], case["smoothing"], case["z_coef"]
    rows = torch.nonzero(s["mask"]).flatten()
    n = max(1, rows.numel())
    nan = float("nan")
    logp = torch.full((T,), nan, dtype=torch.float64, device=DEV)
    lse = torch.full((T,), nan, dtype=torch.float64, device=DEV)
    sums = torch.zeros(4, dtype=torch.float64, device=DEV)
    head = op == "head"
    want = case["grad"]
    if head:
        W = s["W"].double()
        gh = torch.zeros((T, case["D"]), dtype=torch.float64, device=DEV) if want else None
        gw = torch.zeros((V, case["D"]), dtype=torch.float64, device=DEV) if want else None
    else:
        gl = torch.zeros((T, V), dtype=s["logits"].dtype, device=DEV) if want else None
        gl = gl.double() if want and T * V <= 1 << 31 else gl
    step = max(1, min(2048, (1 << 28) // V))
    for r0 in range(0, rows.numel(), step):
        r = rows[r0:r0 + step]
        h = s["hidden"][r].double() if head else None
        z = h @ W.t() if head else s["logits"][r].double()
        y = s["ids"][r].long()
        lp = torch.log_softmax(z, dim=1)
        at = torch.arange(r.numel(), device=DEV)
        l = torch.logsumexp(z, dim=1)
        logp[r], lse[r] = lp[at, y], l
        nll = -lp[at, y]
        smooth = -lp.mean(dim=1) if eps else 0.0 * nll
        sums += torch.stack([((1 - eps) * nll + eps * smooth + zc * l * l).sum(), nll.sum(), smooth.sum(), (l * l).sum()])
        if want:
            target = torch.full_like(z, eps / V)
            target[at, y] += 1.0 - eps
            d = (torch.exp(lp) - target + 2 * zc * l[:, None] * torch.exp(lp)) / n
            if head:
                gh[r] = d @ W
                gw += d.t() @ h
            else:
                gl[r] = d.to(gl.dtype)
    out = dict(logp=logp, lse=lse, loss=sums / n)
    if want and head:
        out["grad_hidden"], out["grad_W"] = gh, gw
    elif want:
        out["grad_logits"] = gl
    return out
