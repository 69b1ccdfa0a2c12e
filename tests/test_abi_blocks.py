"""Host-side refusals of the linear-layer and block-norm entry points: every case fails validation before a device is
touched (no compute without a GPU)."""
import ctypes

import pytest

vp, i32, i64, f32, sz, ci = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_int)
FAKE = 4096          # never dereferenced
NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -8


@pytest.fixture(scope="module")
def lib():
    from paper_2509_06980_b200 import build
    return ctypes.CDLL(build.build())


def test_linear_forward_refuses(lib):
    f = lib.rlf_linear_fwd
    f.argtypes = [vp, i64, i32, i64, vp, i32, vp, ci, ci, ci, vp, i64, vp, ci, vp, vp, vp]

    def call(x=FAKE, T=4, D=64, xs=64, W=FAKE, N=24, b=None, b_dt=0, act=0, gated=0, res=None, rs=24, y=FAKE, dt=0, pre=None, st=None):
        return f(x, T, D, xs, W, N, b, b_dt, act, gated, res, rs, y, dt, pre, st, None)

    assert call(dt=2) == DTYPE and call(b=FAKE, b_dt=7) == DTYPE
    assert call(T=-1) == SHAPE and call(D=0) == SHAPE and call(N=0) == SHAPE and call(D=60, xs=64) == SHAPE and call(xs=56) == SHAPE
    assert call(res=FAKE, rs=23) == SHAPE
    for big in (dict(T=1 << 30), dict(D=1 << 30, xs=1 << 30), dict(N=1 << 29)):
        assert call(**big) == UNSUPPORTED
    assert call(act=5) == UNSUPPORTED and call(act=-1) == UNSUPPORTED and call(gated=2) == UNSUPPORTED
    assert call(x=None) == NULL and call(W=None) == NULL and call(y=None) == NULL
    assert call(x=4104) == ALIGN and call(W=4104) == ALIGN and call(xs=65) == ALIGN and call(y=4097) == ALIGN and call(dt=1, y=4098) == ALIGN
    assert call(res=4097) == ALIGN and call(pre=4097) == ALIGN and call(b=4097) == ALIGN and call(b=4098, b_dt=1) == ALIGN and call(st=4098) == ALIGN
    assert call(T=0, x=None, W=None, y=None) == 0


def test_linear_backward_refuses(lib):
    f = lib.rlf_linear_bwd
    f.argtypes = [vp, ci, i64, vp, vp, i64, i32, i64, vp, i32, ci, ci, vp, vp, ci, vp, ci, vp, sz, vp, vp]

    def call(dy=FAKE, dt=0, ds=24, pre=None, x=FAKE, T=4, D=64, xs=64, W=FAKE, N=24, act=0, gated=0, gx=FAKE, gw=FAKE, w_dt=1, gb=None,
             acc=0, ws=FAKE, wsb=1 << 30, st=None):
        return f(dy, dt, ds, pre, x, T, D, xs, W, N, act, gated, gx, gw, w_dt, gb, acc, ws, wsb, st, None)

    assert call(dt=2) == DTYPE and call(w_dt=3) == DTYPE
    assert call(T=-1) == SHAPE and call(D=12) == SHAPE and call(ds=23) == SHAPE and call(xs=8) == SHAPE
    assert call(act=7) == UNSUPPORTED and call(acc=1, w_dt=0) == UNSUPPORTED
    assert call(dy=None) == NULL and call(x=None) == NULL and call(W=None) == NULL and call(act=2) == NULL and call(gated=1) == NULL
    assert call(dy=4097) == ALIGN and call(x=4104) == ALIGN and call(W=4104) == ALIGN and call(gx=4104) == ALIGN and call(gw=4098) == ALIGN
    assert call(gb=4098) == ALIGN and call(xs=66) == ALIGN and call(act=2, pre=4097) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=4100) == WORKSPACE and call(wsb=64) == WORKSPACE


def test_linear_tuning_refuses(lib):
    f = lib.rlf_tune_linear
    f.argtypes = [ci, ci, ci]
    assert f(4, 0, 0) == SHAPE and f(-1, 0, 0) == SHAPE and f(1, 100, 0) == SHAPE and f(2, 0, 9) == SHAPE and f(2, 0, -1) == SHAPE and f(2, 64, 4) == 0 and f(0, 0, 0) == 0


def test_workspace_sizes(lib):
    lib.rlf_workspace_bytes.restype = sz
    lib.rlf_workspace_bytes.argtypes = [ci, i64, i32, i32, ci]
    w = lib.rlf_workspace_bytes
    assert w(11, 32768, 2560, 4096, 0) >= 2 * 32768 * 2560
    assert w(11, 8191, 1, 4096, 0) < 1 << 24                     # a value head keeps no copy of anything of the batch's size
    assert w(11, 1 << 29, 1 << 12, 64, 0) > 1 << 41              # counted in 64 bits
    assert w(11, -1, 4, 64, 0) == 0 and w(11, 4, 0, 64, 0) == 0


def test_block_norm_forward_refuses(lib):
    f = lib.rlf_block_norm_fwd
    f.argtypes = [vp, i64, vp, ci, i64, i32, vp, vp, ci, vp, vp, ci, ci, vp, ci, f32, f32, f32, vp, vp, vp, vp]

    def call(x=FAKE, xs=64, res=FAKE, dt=0, T=4, D=64, w1=FAKE, b1=None, post=0, w2=FAKE, b2=None, pre=0, w_dt=0, gate=None, form=0,
             alpha=1.0, beta=1.0, eps=1e-6, h=FAKE, y=FAKE, st=None):
        return f(x, xs, res, dt, T, D, w1, b1, post, w2, b2, pre, w_dt, gate, form, alpha, beta, eps, h, y, st, None)

    assert call(dt=2) == DTYPE and call(w_dt=5) == DTYPE
    assert call(T=-1) == SHAPE and call(D=0) == SHAPE and call(xs=63) == SHAPE and call(D=1 << 30, xs=1 << 30) == UNSUPPORTED
    assert call(post=3) == UNSUPPORTED and call(pre=-1) == UNSUPPORTED and call(post=2, pre=2) == UNSUPPORTED and call(form=3) == UNSUPPORTED
    for bad in (float("nan"), float("inf")):
        assert call(alpha=bad) == UNSUPPORTED and call(beta=bad) == UNSUPPORTED and call(eps=bad) == UNSUPPORTED
    assert call(eps=0.0) == UNSUPPORTED
    for k in ("x", "res", "w1", "w2", "h", "y"):
        assert call(**{k: None}) == NULL and call(**{k: 4097}) == ALIGN
    assert call(form=1) == NULL and call(form=2) == NULL and call(form=2, gate=4098) == ALIGN and call(b1=4097) == ALIGN and call(b2=4097) == ALIGN
    assert call(st=4098) == ALIGN and call(T=0, x=None, res=None, w1=None, w2=None, h=None, y=None) == 0


def test_block_norm_backward_refuses(lib):
    f = lib.rlf_block_norm_bwd
    f.argtypes = [vp, vp, vp, i64, vp, ci, i64, i32, vp, vp, ci, vp, ci, ci, vp, ci, f32, f32] + [vp] * 8 + [ci, vp, sz, vp]

    def call(dy=FAKE, dh=None, x=FAKE, xs=64, h=FAKE, dt=0, T=4, D=64, w1=FAKE, b1=None, post=0, w2=FAKE, pre=0, w_dt=0, gate=None, form=0,
             alpha=1.0, beta=1.0, st=FAKE, gx=FAKE, gr=FAKE, gg=None, gw1=FAKE, gb1=None, gw2=FAKE, gb2=None, ws=FAKE, wsb=1 << 30):
        return f(dy, dh, x, xs, h, dt, T, D, w1, b1, post, w2, pre, w_dt, gate, form, alpha, beta, st, gx, gr, gg, gw1, gb1, gw2, gb2, 0, ws,
                 wsb, None)

    assert call(dt=2) == DTYPE and call(T=-1) == SHAPE and call(xs=1) == SHAPE and call(post=9) == UNSUPPORTED
    assert call(post=2) == UNSUPPORTED and call(pre=2, dh=FAKE) == UNSUPPORTED and call(gg=FAKE) == UNSUPPORTED      # gradients of what is not there
    for k in ("dy", "x", "h", "w1", "w2", "st"):
        assert call(**{k: None}) == NULL
    assert call(pre=2, gw2=None, w2=None) == NULL and call(form=1, gg=FAKE) == NULL
    for k in ("dy", "dh", "x", "h", "gx", "gr", "w1", "b1", "w2"):
        assert call(**{k: 4097}) == ALIGN
    for k in ("st", "gw1", "gb1", "gw2", "gb2"):
        assert call(**{k: 4098}) == ALIGN
    assert call(form=2, gate=FAKE, gg=4098) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=4100) == WORKSPACE and call(wsb=64) == WORKSPACE


def test_block_norm_workspace(lib):
    lib.rlf_workspace_bytes.restype = sz
    lib.rlf_workspace_bytes.argtypes = [ci, i64, i32, i32, ci]
    w = lib.rlf_workspace_bytes
    assert 8 * 32768 < w(12, 32768, 0, 2560, 0) < 1 << 27 and w(12, 0, 0, 64, 0) > 0 and w(12, -1, 0, 64, 0) == 0 and w(12, 4, 0, 0, 0) == 0
