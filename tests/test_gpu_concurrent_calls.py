"""Calls of the supervised stage on several streams at once, and replayed graphs of them side by side: the results are
those of the calls one after the other, bit for bit."""
import pytest
import torch

import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def _calls():
    b = gc.binding()
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    z, zo = (3 * r(3000, 30016)).to(BF), (3 * r(4099, 8003))[:, :8000].to(BF)
    H, W = r(700, 512).to(BF), (0.1 * r(20008, 512)).to(BF)
    x, res, w = r(20000, 1024).to(BF), r(20000, 1024).to(BF), (1 + 0.1 * r(1024)).to(BF)
    ids = [torch.randint(0, v, (t,), generator=g, device=DEV, dtype=torch.int32) for t, v in ((3000, 30016), (4099, 8000), (700, 20008))]
    mask = [(torch.rand(t, generator=g, device=DEV) < 0.6).to(torch.uint8) for t in (3000, 4099, 700)]

    def norm():
        y, h, mean, rstd = b.rlf_norm_fwd(x, w, residual=res, kind=b.NORM_LAYER)
        return (y, h, mean, rstd) + b.rlf_norm_bwd(y, h, w, mean, rstd, kind=b.NORM_LAYER, grad_skip=x)[:2]

    return [lambda: b.rlf_cross_entropy_fwd_bwd(z, ids[0], mask[0], z_coef=1e-4),
            lambda: b.rlf_fused_lmhead_cross_entropy(H, W, ids[2], mask[2], label_smoothing=0.1, grad_W_dtype=BF),
            norm,
            lambda: b.rlf_cross_entropy_fwd_bwd(zo, ids[1], mask[1], label_smoothing=0.1),
            lambda: b.rlf_fused_lmhead_cross_entropy(H, W, ids[2], mask[2], want_grad_hidden=False, want_grad_W=False)]


def _same(got, want):
    for a, c in zip(got, want):
        assert (a is None and c is None) or torch.equal(a.nan_to_num(7.0), c.nan_to_num(7.0))


def test_several_streams_at_once():
    calls = _calls()
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = []
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append([c() for _ in range(3)])
        torch.cuda.synchronize()
        for per, w in zip(got, want):
            for o in per:
                _same(o, w)


def test_graphs_replayed_side_by_side():
    calls = _calls()
    want = [c() for c in calls]
    streams, graphs, outs = [], [], []
    for c in calls:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(c())
        streams.append(s)
        graphs.append(g)
    for _ in range(5):
        for o in outs:
            for t in o:
                if t is not None:
                    t.fill_(3.0)
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            _same(o, w)
