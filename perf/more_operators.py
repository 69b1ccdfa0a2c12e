"""The operators around a transformer block of the policy, as they are measured: a linear layer with bias,
activation (plain or gated) and residual in its epilogue, forward and backward, and the norms after one block
and before the next in one pass over the rows, with the block's gate and the residual's scale, forward and
backward.  They are what stands in front of the LM head, and what a value or reward head is made of.

`own = False` computes every operator in elementary torch operations in fp32; `own = True` makes the
library calls of paper_2509_06980_b200.binding.  Both take the same prepared inputs.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
NONE, RELU, SILU, GELU, GELU_TANH = "none", "relu", "silu", "gelu", "gelu_tanh"
RMS, LAYER = "rms", "layer"
ROW, COLUMN = "row", "column"
EPS = 1e-6
DEV = "cuda"


# ---------------------------------------------------------------------------------------------
# cases
def _lin(op, T, D, N, act=NONE, gated=False, bias=False, residual=False, out=BF16, keep=False):
    """T tokens, D inputs, N outputs; keep: the forward pass also leaves what the backward needs."""
    return dict(op=op, T=T, D=D, N=N, act=act, gated=gated, bias=bias, residual=residual, out=out, keep=keep)


def _blk(op, T, D, dt=BF16, w_dt=BF16, post=RMS, pre=RMS, bias=False, gate=NONE, alpha=1.0, beta=1.0, pad=0):
    return dict(op=op, T=T, D=D, dt=dt, w_dt=w_dt, post=post, pre=pre, bias=bias, gate=gate, alpha=alpha, beta=beta,
                pad=pad)


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # eight responses sampled token by token through a gated layer of the 4B-shaped width: the weights are the cost
    add("linear_fwd_decode_gated", _lin("linear_fwd", 8, 2560, 10240, act=SILU, gated=True))
    # a critic's value for each token of one 8192-token response less its prompt, 8B-shaped width, fp32 values
    add("linear_fwd_value_head", _lin("linear_fwd", 8191, 4096, 1, bias=True, out=F32))
    # a reward model's hidden layer: ragged batch, an output width that fills no vector, kept for its backward
    add("linear_fwd_ragged", _lin("linear_fwd", 2047, 1024, 4099, act=GELU, bias=True, keep=True))
    # the training micro-batch of the 4B-shaped recipe (16 responses of 2048 tokens) back to the model's width
    add("linear_fwd_microbatch", _lin("linear_fwd", 32768, 10240, 2560, residual=True))
    # the backward of a short last micro-batch
    add("linear_bwd_short", _lin("linear_bwd", 65, 2560, 2560, act=GELU_TANH, bias=True))
    # the critic's value head again, gradients of its fp32 values
    add("linear_bwd_value_head", _lin("linear_bwd", 8191, 4096, 1, bias=True, out=F32))
    # one 8192-token response through a gated layer of the 8B-shaped width
    add("linear_bwd_gated", _lin("linear_bwd", 8192, 4096, 8192, act=SILU, gated=True))
    # sampling a handful of responses token by token: latency is all that counts
    add("block_norm_fwd_decode", _blk("block_norm_fwd", 8, 2560))
    # the 4B-shaped training micro-batch
    add("block_norm_fwd_microbatch", _blk("block_norm_fwd", 32768, 2560))
    # a small fp32 reward model with layer norms, a ragged batch, a width that fills no vector, a learned gate
    add("block_norm_fwd_layer_odd", _blk("block_norm_fwd", 4999, 1021, dt=F32, w_dt=F32, post=LAYER, pre=LAYER,
                                         bias=True, gate=COLUMN, alpha=1.5))
    # the micro-batch's backward, weight gradients reduced over 32768 rows
    add("block_norm_bwd_microbatch", _blk("block_norm_bwd", 32768, 2560))
    # layer norms with bias and a learned gate over one response less its prompt, fp32 weights beside bf16 rows
    add("block_norm_bwd_layer", _blk("block_norm_bwd", 8191, 4096, w_dt=F32, post=LAYER, pre=LAYER, bias=True,
                                     gate=COLUMN, beta=0.5))
    return c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear_fwd", "linear_bwd", "block_norm_fwd", "block_norm_bwd"])
    if op in ("linear_fwd", "linear_bwd"):
        if rng.random() < 0.2:
            # a value head, or a handful of reward dimensions
            return _lin(op, _log_int(rng, 1, 32768), (_log_int(rng, 64, 8192) + 7) // 8 * 8, rng.randint(1, 4),
                        bias=rng.random() < 0.7, out=F32)
        gated = rng.random() < 0.35
        D = _log_int(rng, 128, 10240)
        D = (D + 63) // 64 * 64 if rng.random() < 0.6 else (D + 7) // 8 * 8
        N = _log_int(rng, 128, 10240)
        if rng.random() < 0.6:
            N = (N + 63) // 64 * 64
        per_token = D * N * (2 if gated else 1) * (2 if op == "linear_bwd" else 1)
        T = _log_int(rng, 1, max(1, min(32768, 32768 * 10240 * 2560 // per_token)))
        act = rng.choice([NONE, RELU, SILU, GELU, GELU_TANH])
        return _lin(op, T, D, N, act=act, gated=gated, bias=rng.random() < 0.5,
                    residual=op == "linear_fwd" and rng.random() < 0.4, keep=op == "linear_fwd" and rng.random() < 0.5)
    D = _log_int(rng, 64, 8192)
    if rng.random() < 0.6:
        D = (D + 63) // 64 * 64
    T = _log_int(rng, 1, max(1, min(65536, 32768 * 2560 // D)))
    post, pre = rng.choice([(RMS, RMS), (LAYER, LAYER), (RMS, NONE), (NONE, RMS), (LAYER, RMS)])
    return _blk(op, T, D, dt=rng.choice([BF16, BF16, F32]), w_dt=rng.choice([BF16, F32]), post=post, pre=pre,
                bias=LAYER in (post, pre) and rng.random() < 0.6, gate=rng.choice([NONE, NONE, COLUMN, ROW]),
                alpha=rng.choice([1.0, 1.0, 0.75]), beta=rng.choice([1.0, 0.5]), pad=rng.choice([0, 0, 8, 3]))


# ---------------------------------------------------------------------------------------------
# inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(shape, g, dt=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dt)


def _prepare_linear(case, g):
    T, D, N = case["T"], case["D"], case["N"]
    rows = 2 * N if case["gated"] else N
    st = dict(case=case, x=_randn((T, D), g, torch.bfloat16), W=_randn((rows, D), g, torch.bfloat16, 1.5 / math.sqrt(D)),
              bias=None, residual=None)
    if case["op"] == "linear_fwd":
        if case["bias"]:
            st["bias"] = _randn((rows,), g, _DT[case["out"]], 0.2)
        if case["residual"]:
            st["residual"] = _randn((T, N), g, _DT[case["out"]], 2.0)
        return st
    st["grad_y"] = _randn((T, N), g, _DT[case["out"]], 1e-3)
    # the layer's output before its activation, as the forward pass left it
    st["pre"] = _randn((T, rows), g, torch.bfloat16, 1.5) if case["act"] != NONE or case["gated"] else None
    return st


def _prepare_block(case, g):
    T, D, dt, w_dt = case["T"], case["D"], _DT[case["dt"]], _DT[case["w_dt"]]

    def vector(there, mean, spread):
        return (mean + spread * _randn((D,), g)).to(w_dt) if there else None

    post, pre = case["post"] != NONE, case["pre"] != NONE
    st = dict(case=case, post_weight=vector(post, 1.0, 0.2), pre_weight=vector(pre, 1.0, 0.2),
              post_bias=vector(post and case["bias"], 0.0, 0.1), pre_bias=vector(pre and case["bias"], 0.0, 0.1), gate=None)
    if case["gate"] == COLUMN:
        st["gate"] = vector(True, 0.5, 0.3)
    elif case["gate"] == ROW:
        st["gate"] = torch.rand((T,), generator=g, device=DEV)
    # a block's output and the residual stream: a few columns far larger than the others, a small offset
    x = _randn((T, D + case["pad"]), g, torch.float32, 1.0) + 0.1
    st["x"] = x.to(dt)[:, :D]
    r = _randn((T, D), g, torch.float32, 2.0) + 0.25
    r[:, :: max(1, D // 7)] *= 8.0
    if case["op"] == "block_norm_fwd":
        st["residual"] = r.to(dt)
        return st
    st["h"] = r.to(dt)
    st["grad_y"] = _randn((T, D), g, dt, 1e-3) if pre else None
    st["grad_h"] = _randn((T, D), g, dt, 1e-3)
    # statistics as the forward pass leaves them: mean and 1 / spread of the block's output, then of the stream
    stats = torch.zeros((4, T), device=DEV)
    stats[1] = stats[3] = 1.0
    for at, kind, rows in ((0, case["post"], st["x"]), (2, case["pre"], st["h"])):
        if kind == NONE:
            continue
        f = rows.float()
        if kind == LAYER:
            stats[at] = f.mean(dim=1)
            f = f - stats[at][:, None]
        stats[at + 1] = torch.rsqrt((f * f).mean(dim=1) + EPS)
    st["stats"] = stats
    return st


def prepare(case, seed):
    g = _gen(seed)
    return _prepare_linear(case, g) if case["op"].startswith("linear") else _prepare_block(case, g)


# ---------------------------------------------------------------------------------------------
# plain forms (fp32, elementary operations)
_ROOT = math.sqrt(2.0 / math.pi)


def _act(z, act):
    if act == RELU:
        return torch.clamp(z, min=0.0)
    if act == SILU:
        return z * torch.sigmoid(z)
    if act == GELU:
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if act == GELU_TANH:
        return z * torch.sigmoid(2.0 * _ROOT * (z + 0.044715 * z * z * z))
    return z


def _act_slope(z, act):
    if act == RELU:
        return (z > 0).to(z.dtype)
    if act == SILU:
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    if act == GELU:
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == GELU_TANH:
        s = torch.sigmoid(2.0 * _ROOT * (z + 0.044715 * z * z * z))
        return s + z * s * (1.0 - s) * 2.0 * _ROOT * (1.0 + 3.0 * 0.044715 * z * z)
    return torch.ones_like(z)


def _linear_fwd_plain(s):
    case = s["case"]
    z = s["x"].float() @ s["W"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z[:, :case["N"]], case["act"])
    if case["gated"]:
        y = y * z[:, case["N"]:]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(y=y.to(_DT[case["out"]]))
    if case["keep"]:
        out["pre"] = z.to(torch.bfloat16)
    return out


def _linear_bwd_plain(s):
    case = s["case"]
    N, act = case["N"], case["act"]
    g = s["grad_y"].float()
    if s["pre"] is not None:
        z = s["pre"].float()
        if case["gated"]:
            g = torch.cat([g * z[:, N:] * _act_slope(z[:, :N], act), g * _act(z[:, :N], act)], dim=1)
        else:
            g = g * _act_slope(z, act)
    out = dict(grad_x=(g @ s["W"].float()).to(torch.bfloat16), grad_W=(g.t() @ s["x"].float()).to(torch.bfloat16))
    if case["bias"]:
        out["grad_bias"] = g.sum(dim=0)
    return out


def _normed(rows, kind, weight, bias):
    """-> the normed rows (the rows themselves without a norm), their mean and 1 / spread"""
    T = rows.shape[0]
    if kind == NONE:
        return rows, torch.zeros(T, device=DEV), torch.ones(T, device=DEV)
    mean = rows.mean(dim=1) if kind == LAYER else torch.zeros(T, device=DEV)
    c = rows - mean[:, None]
    rstd = torch.rsqrt((c * c).mean(dim=1) + EPS)
    y = c * rstd[:, None] * weight.float()
    return (y if bias is None else y + bias.float()), mean, rstd


def _gate_rows(s):
    """the gate times the branch's scale, as something that multiplies [T, D]"""
    case = s["case"]
    if case["gate"] == COLUMN:
        return case["beta"] * s["gate"].float()[None, :]
    if case["gate"] == ROW:
        return case["beta"] * s["gate"][:, None]
    return case["beta"]


def _block_fwd_plain(s):
    case = s["case"]
    n, m1, r1 = _normed(s["x"].float(), case["post"], s["post_weight"], s["post_bias"])
    h = case["alpha"] * s["residual"].float() + _gate_rows(s) * n
    y, m2, r2 = _normed(h, case["pre"], s["pre_weight"], s["pre_bias"])
    out = dict(h=h.to(s["x"].dtype), stats=torch.stack([m1, r1, m2, r2]))
    if case["pre"] != NONE:
        out["y"] = y.to(s["x"].dtype)
    return out


def _norm_grad(g, rows, kind, weight, mean, rstd):
    """-> gradient of the rows, and the normed rows before their weight"""
    xh = (rows - mean[:, None]) * rstd[:, None]
    q = g * weight.float()
    d = q - xh * (q * xh).mean(dim=1, keepdim=True)
    if kind == LAYER:
        d = d - q.mean(dim=1, keepdim=True)
    return d * rstd[:, None], xh


def _block_bwd_plain(s):
    case, st = s["case"], s["stats"]
    dt = s["x"].dtype
    out = {}
    gh = s["grad_h"].float()
    if case["pre"] != NONE:
        gy = s["grad_y"].float()
        d, hh = _norm_grad(gy, s["h"].float(), case["pre"], s["pre_weight"], st[2], st[3])
        gh = gh + d
        out["grad_pre_weight"] = (gy * hh).sum(dim=0)
        if case["bias"]:
            out["grad_pre_bias"] = gy.sum(dim=0)
    out["grad_residual"] = (case["alpha"] * gh).to(dt)
    x = s["x"].float()
    gn = _gate_rows(s) * gh
    if case["post"] != NONE:
        d, xh = _norm_grad(gn, x, case["post"], s["post_weight"], st[0], st[1])
        out["grad_x"] = d.to(dt)
        out["grad_post_weight"] = (gn * xh).sum(dim=0)
        if case["bias"]:
            out["grad_post_bias"] = gn.sum(dim=0)
        n = xh * s["post_weight"].float()
        if s["post_bias"] is not None:
            n = n + s["post_bias"].float()
    else:
        out["grad_x"] = gn.to(dt)
        n = x
    if case["gate"] != NONE:
        out["grad_gate"] = (case["beta"] * gh * n).sum(dim=0 if case["gate"] == COLUMN else 1)
    return out


# ---------------------------------------------------------------------------------------------
# the library's calls
def _own(s):
    from paper_2509_06980_b200 import binding as rlf

    case = s["case"]
    op = case["op"]
    if op in ("linear_fwd", "linear_bwd"):
        act = {NONE: rlf.ACT_NONE, RELU: rlf.ACT_RELU, SILU: rlf.ACT_SILU, GELU: rlf.ACT_GELU,
               GELU_TANH: rlf.ACT_GELU_TANH}[case["act"]]
        if op == "linear_fwd":
            y, pre = rlf.rlf_linear_fwd(s["x"], s["W"], bias=s["bias"], act=act, gated=case["gated"], residual=s["residual"],
                                        out_dtype=_DT[case["out"]], want_pre=case["keep"])
            return dict(y=y, pre=pre) if case["keep"] else dict(y=y)
        gx, gw, gb = rlf.rlf_linear_bwd(s["grad_y"], s["x"], s["W"], pre=s["pre"], act=act, gated=case["gated"],
                                        grad_W_dtype=torch.bfloat16, want_grad_bias=case["bias"])
        out = dict(grad_x=gx, grad_W=gw)
        if gb is not None:
            out["grad_bias"] = gb
        return out
    kinds = {NONE: rlf.NORM_NONE, RMS: rlf.NORM_RMS, LAYER: rlf.NORM_LAYER}
    form = dict(post_kind=kinds[case["post"]], pre_kind=kinds[case["pre"]], alpha=case["alpha"], beta=case["beta"],
                gate=s["gate"], gate_form={NONE: rlf.GATE_NONE, COLUMN: rlf.GATE_COLUMN, ROW: rlf.GATE_ROW}[case["gate"]])
    if op == "block_norm_fwd":
        h, y, stats = rlf.rlf_block_norm_fwd(s["x"], s["residual"], post_weight=s["post_weight"], post_bias=s["post_bias"],
                                             pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], eps=EPS, **form)
        out = dict(h=h, stats=stats)
        if y is not None:
            out["y"] = y
        return out
    g = rlf.rlf_block_norm_bwd(s["grad_y"], s["grad_h"], s["x"], s["h"], s["stats"], post_weight=s["post_weight"],
                               post_bias=s["post_bias"], pre_weight=s["pre_weight"], want_grad_bias=case["bias"], **form)
    return {k: v for k, v in g.items() if v is not None}


_PLAIN = dict(linear_fwd=_linear_fwd_plain, linear_bwd=_linear_bwd_plain, block_norm_fwd=_block_fwd_plain,
              block_norm_bwd=_block_bwd_plain)


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
def work(case):
    op, T, D = case["op"], case["T"], case["D"]
    if op in ("linear_fwd", "linear_bwd"):
        N, osz = case["N"], 2 if case["out"] == BF16 else 4
        rows = 2 * N if case["gated"] else N
        nbytes = 2 * (T * D + rows * D) + T * N * osz
        if op == "linear_fwd":
            nbytes += (rows * osz if case["bias"] else 0) + (T * N * osz if case["residual"] else 0)
            nbytes += 2 * T * rows if case["keep"] else 0
            return dict(bytes=nbytes, flops=2 * T * D * rows)
        nbytes += 2 * (T * D + rows * D) + (4 * rows if case["bias"] else 0)
        nbytes += 2 * T * rows if case["act"] != NONE or case["gated"] else 0
        return dict(bytes=nbytes, flops=4 * T * D * rows)
    esz, wsz = 2 if case["dt"] == BF16 else 4, 2 if case["w_dt"] == BF16 else 4
    norms = (case["post"] != NONE) + (case["pre"] != NONE)
    vectors = norms * (2 if case["bias"] else 1) + (case["gate"] == COLUMN)
    small = 16 * T + vectors * D * wsz + (4 * T if case["gate"] == ROW else 0)
    if op == "block_norm_fwd":
        return dict(bytes=T * D * esz * (4 if case["pre"] != NONE else 3) + small, flops=(4 + 6 * norms) * T * D)
    small += vectors * D * 4 + (4 * T if case["gate"] == ROW else 0)
    return dict(bytes=T * D * esz * (6 if case["pre"] != NONE else 4) + small, flops=(4 + 12 * norms) * T * D)


# ---------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
def _phi(z):
    return 0.5 * (1.0 + torch.special.erf(z * math.sqrt(0.5)))


def _value_and_slope64(z, act):
    """An activation and its derivative."""
    if act == NONE:
        return z, torch.ones_like(z)
    if act == RELU:
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).double()
    if act == SILU:
        e = torch.exp(-z)
        return z / (1 + e), (1 + e + z * e) / (1 + e) ** 2
    if act == GELU:
        return z * _phi(z), _phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c, k = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(c * (z + k * z ** 3))
    return z * (1 + t) / 2, (1 + t) / 2 + z / 2 * (1 - t * t) * c * (1 + 3 * k * z * z)


def exact(case, seed):
    s = prepare(case, seed)
    op, T, D = case["op"], case["T"], case["D"]
    if op == "linear_fwd":
        N = case["N"]
        z = torch.einsum("td,nd->tn", s["x"].double(), s["W"].double())
        if s["bias"] is not None:
            z += s["bias"].double()
        y = _value_and_slope64(z[:, :N], case["act"])[0]
        if case["gated"]:
            y = y * z[:, N:]
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return dict(y=y, pre=z) if case["keep"] else dict(y=y)
    if op == "linear_bwd":
        N = case["N"]
        g = s["grad_y"].double()
        if s["pre"] is not None:
            value, slope = _value_and_slope64(s["pre"][:, :N].double(), case["act"])
            if case["gated"]:
                up = s["pre"][:, N:].double()
                g = torch.cat([g * slope * up, g * value], dim=1)
            else:
                g = g * slope
        out = dict(grad_x=torch.einsum("tn,nd->td", g, s["W"].double()),
                   grad_W=torch.einsum("tn,td->nd", g, s["x"].double()))
        if case["bias"]:
            out["grad_bias"] = g.sum(dim=0)
        return out

    def wide(name, default):
        v = s[name]
        return torch.full((D,), default, dtype=torch.float64, device=DEV) if v is None else v.double()

    gate = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    if case["gate"] != NONE:
        gate = s["gate"].double().reshape((1, D) if case["gate"] == COLUMN else (T, 1))
    gate = gate * case["beta"]
    w1, b1, w2, b2 = wide("post_weight", 1.0), wide("post_bias", 0.0), wide("pre_weight", 1.0), wide("pre_bias", 0.0)
    x = s["x"].double()

    def unit(rows, kind):
        mu = rows.sum(dim=1) / D if kind == LAYER else torch.zeros(T, dtype=torch.float64, device=DEV)
        if kind == NONE:
            return rows, mu, torch.ones_like(mu)
        c = rows - mu[:, None]
        r = 1.0 / torch.sqrt((c ** 2).sum(dim=1) / D + EPS)
        return c * r[:, None], mu, r

    if op == "block_norm_fwd":
        xh, m1, r1 = unit(x, case["post"])
        h = case["alpha"] * s["residual"].double() + gate * (xh * w1 + b1)
        hh, m2, r2 = unit(h, case["pre"])
        out = dict(h=h, stats=torch.stack([m1, r1, m2, r2]))
        if case["pre"] != NONE:
            out["y"] = hh * w2 + b2
        return out

    st = s["stats"].double()
    xh = (x - st[0][:, None]) * st[1][:, None]
    gh = s["grad_h"].double()
    out = {}

    def back(g, w, unit_rows, r, kind):
        q = g * w
        inner = torch.einsum("td,td->t", q, unit_rows) / D
        shift = q.sum(dim=1) / D if kind == LAYER else torch.zeros_like(inner)
        return (q - shift[:, None] - unit_rows * inner[:, None]) * r[:, None]

    if case["pre"] != NONE:
        gy = s["grad_y"].double()
        hh = (s["h"].double() - st[2][:, None]) * st[3][:, None]
        gh = gh + back(gy, w2, hh, st[3], case["pre"])
        out["grad_pre_weight"] = torch.einsum("td,td->d", gy, hh)
        if case["bias"]:
            out["grad_pre_bias"] = gy.sum(dim=0)
    out["grad_residual"] = gh * case["alpha"]
    gn = gh * gate
    if case["post"] != NONE:
        out["grad_x"] = back(gn, w1, xh, st[1], case["post"])
        out["grad_post_weight"] = torch.einsum("td,td->d", gn, xh)
        if case["bias"]:
            out["grad_post_bias"] = gn.sum(dim=0)
    else:
        out["grad_x"] = gn
    if case["gate"] != NONE:
        n = gh * (xh * w1 + b1) * case["beta"]
        out["grad_gate"] = n.sum(dim=0) if case["gate"] == COLUMN else n.sum(dim=1)
    return out
