"""The supervised operators run together as a training step uses them (mask, final norm with the residual stream,
cross entropy through the head, norm backward) on the GPU, against the fp64 definitions."""
import numpy as np
import pytest
import torch

from oracle import operators64 as o64
from oracle import rlf_oracle as orc
from paper_2509_06980_b200 import sharded, synth
import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _batch():
    spec = synth.scaled(synth.SPECS[3], V=2048, D=128, w_std=0.3, len_lo=20, len_hi=40, spans_lo=1, spans_hi=2, obs_lo=2, obs_hi=4)
    tok = synth.make_tokens(spec)
    T = len(tok.ids)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x, res = r(T, spec.D).bfloat16(), r(T, spec.D).bfloat16()
    W, w, b = (0.3 * r(spec.V, spec.D)).bfloat16(), (1 + 0.2 * r(spec.D)).bfloat16(), (0.1 * r(spec.D)).bfloat16()
    return spec, tok, torch.from_numpy(tok.ids).to(DEV), torch.from_numpy(tok.cu_seqlens).to(DEV), x, res, W, w, b


def _close(got, want, tol, what):
    got = got.double().cpu().numpy()
    err = np.abs(got - want).max() / np.abs(want).max()
    assert err <= tol, (what, err)


@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
def test_step_against_the_definitions(layer):
    """Every stage takes the previous one's bf16 result, as the definitions here do, so the stages' own bounds add up: the
    normed row is off by one rounding (2^-8); a logit by that times sum |h w| of about 0.3 sqrt(128) standard deviations;
    gradients by a handful of roundings (2^-8 each) of their largest entries: 2^-5 of the tensor's largest value."""
    b = gc.binding()
    spec, tok, ids, cu, x, res, W, w, bias = _batch()
    out = sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, hidden=x, residual=res, W=W, norm_weight=w,
                                   norm_bias=bias if layer else None, norm_kind=b.NORM_LAYER if layer else b.NORM_RMS,
                                   label_smoothing=0.1, z_coef=1e-4)
    f = lambda t: t.double().cpu().numpy()
    mask, _, n = orc.build_loss_mask(tok.ids, tok.cu_seqlens, spec.open_id, spec.close_id)
    assert np.array_equal(out["mask"].cpu().numpy(), mask) and int(out["n_global"]) == n
    y, h, mu, r = o64.norm(f(x), f(w), f(bias) if layer else None, f(res), layer, 1e-6)
    y16 = f(torch.from_numpy(y).bfloat16())
    q = o64.fused_cross_entropy(y16, f(W), tok.ids, mask, 0.1, 1e-4)
    live = mask != 0
    assert np.array_equal(np.isnan(out["logp"].cpu().numpy()), ~live)
    # rows whose normed values round the other way differ by a step (2^-7) in single entries
    tol = 2.0 ** -7 * np.abs(y16).max() * np.abs(f(W)).max() * 4
    assert np.abs(out["logp"].double().cpu().numpy() - q["logp"])[live].max() <= tol
    assert np.abs(f(out["loss"]) - q["loss"]).max() <= 2.0 ** -7 * np.abs(q["loss"]).max()
    h16 = f(torch.from_numpy(h).bfloat16())
    gx, gw, gb = o64.norm_grad(q["grad_hidden"], h16, f(w), mu, r, layer)
    _close(out["grad_W"], q["grad_W"], 2.0 ** -5, "grad_W")
    _close(out["grad_hidden"], gx, 2.0 ** -5, "grad_hidden")
    _close(out["grad_norm_weight"], gw, 2.0 ** -5, "grad_norm_weight")
    if layer:
        _close(out["grad_norm_bias"], gb, 2.0 ** -5, "grad_norm_bias")
    assert not out["grad_hidden"][torch.from_numpy(~live).to(DEV)].any()


def test_shards_add_up_to_the_whole_batch():
    """The parts of two ranks run one after the other on one GPU, against the batch's count."""
    spec, tok, ids, cu, x, res, W, w, _ = _batch()
    kw = dict(W=W, norm_weight=w, label_smoothing=0.1)
    whole = sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, hidden=x, residual=res, **kw)
    gw, gnw, loss = 0.0, 0.0, 0.0
    for part in sharded.plan_shards(tok.cu_seqlens, 1, 2):
        cu_k, t_k, _ = sharded.take_shard(part, tok.cu_seqlens, {"ids": tok.ids, "rows": np.arange(len(tok.ids))}, {})
        rows = torch.from_numpy(t_k["rows"]).to(DEV)
        o = sharded.sharded_sft_step(torch.from_numpy(t_k["ids"]).to(DEV), torch.from_numpy(cu_k).to(DEV), spec.open_id,
                                     spec.close_id, hidden=x[rows], residual=res[rows], n_global=whole["n_global"], **kw)
        gw, gnw, loss = gw + o["grad_W"], gnw + o["grad_norm_weight"], loss + o["loss"]
        # (row results: the same but for the order of the sums over the vocabulary, which the number of rows decides)
        assert torch.allclose(o["logp"].nan_to_num(0.0), whole["logp"][rows].nan_to_num(0.0), atol=2e-5)
        d = (o["grad_hidden"].float() - whole["grad_hidden"][rows].float()).abs().max()
        assert d <= 2.0 ** -6 * whole["grad_hidden"].float().abs().max()
    assert torch.allclose(loss, whole["loss"], rtol=1e-6)
    assert (gw - whole["grad_W"]).abs().max() <= 2.0 ** -7 * whole["grad_W"].abs().max()
    assert (gnw - whole["grad_norm_weight"]).abs().max() <= 2.0 ** -6 * whole["grad_norm_weight"].abs().max()


def test_logits_path_and_head_path_agree():
    spec, tok, ids, cu, x, _, W, _, _ = _batch()
    a = sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, hidden=x, W=W, label_smoothing=0.1, z_coef=1e-3)
    c = sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, logits=x.float() @ W.float().t(), label_smoothing=0.1,
                                 z_coef=1e-3)
    assert torch.allclose(a["loss"], c["loss"], rtol=1e-5)
    gh = c["grad_logits"] @ W.float()
    assert (a["grad_hidden"].float() - gh).abs().max() <= 2.0 ** -6 * gh.abs().max()


def test_step_captured_and_replayed():
    spec, tok, ids, cu, x, res, W, w, _ = _batch()
    call = lambda: sharded.sharded_sft_step(ids, cu, spec.open_id, spec.close_id, hidden=x, residual=res, W=W, norm_weight=w)
    ref = call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    x.mul_(-1)
    g.replay()
    x.mul_(-1)
    g.replay()
    torch.cuda.synchronize()
    for k in ref:
        assert torch.equal(out[k].nan_to_num(5.0), ref[k].nan_to_num(5.0)), k
