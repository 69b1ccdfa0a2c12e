"""A feed-forward block in front of the LM head, forward and backward, as a training step runs it: norm, gated linear layer,
linear layer, norm with gate and residual and the norm behind it in one call, cross entropy through the head, and back.  Every
gradient is compared with fp64 autograd of the same formulas on the same bf16 weights.

Tolerance: intermediate activations and gradients are bf16 (a random error of up to half a step, 2^-8 of the value, rms 2^-8 / sqrt 3)
at nine places on the way to the first gradient; errors add in squares, so a gradient is off by about 3 x 2^-8 / sqrt 3 = 0.7 % of
its size (Frobenius norm); the bound is 4 times that, and a wrong term shows as tens of per cent."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
EPS = 1e-6


def _weights(D, F, V, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s, k=1.0: (torch.randn(*s, generator=g, device=DEV) * k)
    return dict(n0=(1 + 0.1 * r(D)).to(BF), up=r(2 * F, D, k=D ** -0.5).to(BF), up_b=r(2 * F, k=0.1).to(BF), down=r(D, F, k=F ** -0.5).to(BF),
                down_b=r(D, k=0.1).to(BF), n1=(1 + 0.1 * r(D)).to(BF), gate=(0.5 + 0.2 * r(D)).to(BF), n2=(1 + 0.1 * r(D)).to(BF),
                head=r(V, D, k=2.0 * D ** -0.5).to(BF))


def step(b, w, x, ids, mask, alpha=1.0, beta=1.0):
    """-> (loss, dict of gradients)"""
    n, _, _, r0 = b.rlf_norm_fwd(x, w["n0"], eps=EPS)
    a, pre = b.rlf_linear_fwd(n, w["up"], bias=w["up_b"], act=b.ACT_SILU, gated=True, want_pre=True)
    o, _ = b.rlf_linear_fwd(a, w["down"], bias=w["down_b"])
    form = dict(gate=w["gate"], gate_form=b.GATE_COLUMN, alpha=alpha, beta=beta)
    h, y, stats = b.rlf_block_norm_fwd(o, x, post_weight=w["n1"], pre_weight=w["n2"], eps=EPS, **form)
    _, _, loss, gy, g_head = b.rlf_fused_lmhead_cross_entropy(y, w["head"], ids, mask, grad_W_dtype=torch.float32)
    k = b.rlf_block_norm_bwd(gy, None, o, h, stats, post_weight=w["n1"], pre_weight=w["n2"], **form)
    ga, g_down, g_down_b = b.rlf_linear_bwd(k["grad_x"], a, w["down"], want_grad_bias=True)
    gn, g_up, g_up_b = b.rlf_linear_bwd(ga, n, w["up"], pre=pre, act=b.ACT_SILU, gated=True, want_grad_bias=True)
    gx, g_n0, _ = b.rlf_norm_bwd(gn, x, w["n0"], None, r0, grad_skip=k["grad_residual"])
    return loss, dict(x=gx, n0=g_n0, up=g_up, up_b=g_up_b, down=g_down, down_b=g_down_b, n1=k["grad_post_weight"], n2=k["grad_pre_weight"],
                      gate=k["grad_gate"], head=g_head)


def reference(w, x, ids, mask, alpha, beta):
    p = {k: v.double().requires_grad_() for k, v in dict(w, x=x).items()}
    rms = lambda v, s: v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * s
    z = rms(p["x"], p["n0"]) @ p["up"].t() + p["up_b"]
    F = p["down"].shape[1]
    a = torch.nn.functional.silu(z[:, :F]) * z[:, F:]
    h = alpha * p["x"] + beta * p["gate"] * rms(a @ p["down"].t() + p["down_b"], p["n1"])
    lp = torch.log_softmax(rms(h, p["n2"]) @ p["head"].t(), dim=1)
    live = mask != 0
    loss = -lp[torch.arange(len(ids), device=DEV), ids.long()][live].sum() / live.sum()
    loss.backward()
    return loss.item(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("T,D,F,V,alpha,beta", [(5, 128, 192, 512, 1.0, 1.0), (300, 256, 520, 1024, 0.75, 0.5), (1100, 512, 1000, 2048, 1.0, 1.0)])
def test_block_in_front_of_the_head(T, D, F, V, alpha, beta):
    b = gc.binding()
    w = _weights(D, F, V, T)
    x = torch.randn(T, D, device=DEV).to(BF)
    ids = torch.randint(0, V, (T,), device=DEV, dtype=torch.int32)
    mask = (torch.rand(T, device=DEV) < 0.7).to(torch.uint8)
    mask[0] = 1
    loss, got = step(b, w, x, ids, mask, alpha, beta)
    want_loss, want = reference(w, x, ids, mask, alpha, beta)
    assert abs(loss[0].item() - want_loss) < 0.02 * abs(want_loss)
    for k, g in got.items():
        err = (g.double() - want[k]).norm() / want[k].norm()
        assert err < 4 * 0.007, (k, err.item())
    # captured and replayed beside an eager run of the same step, on the same weights
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b, w, x, ids, mask, alpha, beta)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        _, kept = step(b, w, x, ids, mask, alpha, beta)
    _, again = step(b, w, x, ids, mask, alpha, beta)
    graph.replay()
    torch.cuda.synchronize()
    for k in got:
        assert torch.equal(kept[k], again[k]) and torch.equal(got[k], again[k]), k


def test_one_token_at_a_time_gives_the_rows_of_the_batch():
    """Decoding: each row through the streamed forms against the same rows in one batch, to two roundings of each output."""
    b = gc.binding()
    T, D, F = 300, 256, 264
    w = _weights(D, F, 64, 3)
    x = torch.randn(T, D, device=DEV).to(BF)

    def block(rows):
        n, _, _, _ = b.rlf_norm_fwd(rows, w["n0"], eps=EPS)
        a, _ = b.rlf_linear_fwd(n, w["up"], act=b.ACT_SILU, gated=True)
        o, _ = b.rlf_linear_fwd(a, w["down"])
        return b.rlf_block_norm_fwd(o, rows, post_weight=w["n1"], pre_weight=w["n2"], eps=EPS)[1]

    whole = block(x).float()
    for at in (0, 1, 150, 299):
        one = block(x[at:at + 1]).float()
        assert ((one[0] - whole[at]).norm() / whole[at].norm()).item() < 4 * 2.0 ** -8
    few = block(x[100:117]).float()
    assert ((few - whole[100:117]).norm() / whole[100:117].norm()).item() < 4 * 2.0 ** -8


def test_two_streams_at_once():
    """The same step on two streams at the same time, several times over: bit-identical to a single run."""
    b = gc.binding()
    w = _weights(256, 520, 1024, 1)
    x = torch.randn(400, 256, device=DEV).to(BF)
    ids = torch.randint(0, 1024, (400,), device=DEV, dtype=torch.int32)
    mask = torch.ones(400, device=DEV, dtype=torch.uint8)
    _, want = step(b, w, x, ids, mask)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(step(b, w, x, ids, mask)[1])
    torch.cuda.synchronize()
    for g in got:
        for k in want:
            assert torch.equal(g[k], want[k]), k
