"""The layers in front of the head and the norms around them, several calls at once: two captured steps replayed side by side while
a third runs eagerly, each on a stream and with workspaces of its own.  Every result is bit-identical to that of a step alone."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def _inputs(T, D, F, N, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s, k=1.0: (torch.randn(*s, generator=g, device=DEV) * k).to(BF)
    return dict(x=r(T, D), up=r(2 * F, D, k=D ** -0.5), down=r(D, F, k=F ** -0.5), n1=1 + r(D, k=0.1), n2=1 + r(D, k=0.1), head=r(N, D, k=D ** -0.5),
                gate=r(2 * N, D, k=D ** -0.5), dv=r(T, N))


def _step(b, w):
    a, pre = b.rlf_linear_fwd(w["x"], w["up"], act=b.ACT_SILU, gated=True, want_pre=True)
    o, _ = b.rlf_linear_fwd(a, w["down"])
    norms = dict(post_weight=w["n1"], pre_weight=w["n2"])
    h, y, stats = b.rlf_block_norm_fwd(o, w["x"], **norms)
    v, _ = b.rlf_linear_fwd(y, w["head"], out_dtype=torch.float32)
    u, pre_u = b.rlf_linear_fwd(y, w["gate"], act=b.ACT_GELU, gated=True, want_pre=True)
    gy, g_head, g_head_b = b.rlf_linear_bwd(w["dv"], y, w["head"], want_grad_bias=True)
    gy2, g_gate, g_gate_b = b.rlf_linear_bwd(w["dv"], y, w["gate"], pre=pre_u, act=b.ACT_GELU, gated=True, want_grad_bias=True)
    k = b.rlf_block_norm_bwd(gy, gy2, o, h, stats, **norms)
    ga, g_down, _ = b.rlf_linear_bwd(k["grad_x"], a, w["down"])
    gx, g_up, _ = b.rlf_linear_bwd(ga, w["x"], w["up"], pre=pre, act=b.ACT_SILU, gated=True)
    return [v, u, g_head, g_head_b, g_gate, g_gate_b, k["grad_post_weight"], k["grad_pre_weight"], g_down, gx, g_up]


@pytest.mark.parametrize("sizes", [((8, 256, 520, 1), (8, 256, 520, 2)), ((1500, 256, 520, 1), (70, 512, 264, 2)), ((3000, 512, 1000, 2), (2000, 264, 1032, 1))])
def test_two_graphs_and_an_eager_step(sizes):
    b = gc.binding()
    steps = [_inputs(*s, seed=i) for i, s in enumerate(sizes)]
    third = _inputs(*sizes[0], seed=9)
    want = [[t.clone() for t in _step(b, w)] for w in steps + [third]]
    torch.cuda.synchronize()
    graphs, kept = [], []
    for w in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept.append(_step(b, w))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(6):
        for outs in kept:
            for t in outs:
                t.fill_(3.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = _step(b, third)
        torch.cuda.synchronize()
        for outs, ref in zip(kept + [eager], want):
            assert all(torch.equal(p, q) for p, q in zip(outs, ref))
