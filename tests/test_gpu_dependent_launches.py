"""Calls whose launches follow one another without a gap, each reading what the one before it wrote: a hidden layer and a value head on
it, forward and backward, over the same activations' buffers again and again without a pause, eagerly and as a graph, against the
same calls with a synchronisation after each."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("T,D,N", [(1, 128, 1), (8, 512, 1), (100, 256, 2), (700, 512, 1), (2500, 256, 3)])
def test_values_of_what_was_just_written(T, D, N):
    b = gc.binding()
    g = torch.Generator(device=DEV)
    g.manual_seed(T + D + N)
    r = lambda *s, k=1.0: (torch.randn(*s, generator=g, device=DEV) * k).to(BF)
    up, head, dy, xs = r(D, D, k=D ** -0.5), r(N, D, k=D ** -0.5), r(T, N).float(), r(24, T, D)
    h, z, gh, gx = (torch.zeros(T, D, dtype=BF, device=DEV) for _ in range(4))
    bwd_ws = [b.new_workspace(b.FN_LINEAR_BWD, T, n, D) for n in (N, D)]

    def outputs():
        n = len(xs)
        return dict(first=torch.zeros(n, T, N, device=DEV), second=torch.zeros(n, T, N, device=DEV), head=torch.zeros(n, N, D, device=DEV),
                    head_b=torch.zeros(n, N, device=DEV), up=torch.zeros(n, D, D, device=DEV), up_b=torch.zeros(n, D, device=DEV))

    def run(out, pause=lambda: None):
        for i, x in enumerate(xs):
            b.rlf_linear_fwd(x, up, act=b.ACT_SILU, y_out=h, pre_out=z)
            pause()
            b.rlf_linear_fwd(h, head, y_out=out["first"][i])
            pause()
            b.rlf_linear_bwd(dy, h, head, grad_x=gh, grad_W=out["head"][i], grad_bias=out["head_b"][i], workspace=bwd_ws[0])
            pause()
            b.rlf_linear_bwd(gh, x, up, pre=z, act=b.ACT_SILU, grad_x=gx, grad_W=out["up"][i], grad_bias=out["up_b"][i], workspace=bwd_ws[1])
            pause()
            b.rlf_linear_fwd(gx, up, act=b.ACT_GELU, residual=h, y_out=h)          # (onto the hidden state that was read above)
            pause()
            b.rlf_linear_fwd(h, head, y_out=out["second"][i])
            pause()
        return out

    want = run(outputs(), torch.cuda.synchronize)
    kept = outputs()
    run(kept)                                                   # (warm-up of the capture, and the eager run)
    torch.cuda.synchronize()
    assert all(torch.equal(kept[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(kept)
    for _ in range(3):
        for t in kept.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(kept[k], want[k]) for k in want)
