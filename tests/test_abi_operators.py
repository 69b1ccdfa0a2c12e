"""Host-side refusals of the cross-entropy and norm entry points: every case fails validation before a device
is touched (no compute without a GPU)."""
import ctypes

import pytest

vp, i32, i64, f32, sz, ci = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_int)
FAKE = 4096          # never dereferenced
NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -8


@pytest.fixture(scope="module")
def lib():
    from paper_2509_06980_b200 import build
    return ctypes.CDLL(build.build())


def test_norm_forward_refuses(lib):
    f = lib.rlf_norm_fwd
    f.argtypes = [vp, vp, ci, i64, i32, i64, vp, vp, ci, ci, f32, vp, vp, vp, vp, vp]

    def call(x=FAKE, res=None, dt=0, T=4, D=64, stride=64, w=FAKE, b=None, w_dt=0, kind=0, eps=1e-6, s=None, y=FAKE,
             mean=None, rstd=None):
        return f(x, res, dt, T, D, stride, w, b, w_dt, kind, eps, s, y, mean, rstd, None)

    assert call(dt=2) == DTYPE and call(w_dt=-1) == DTYPE
    assert call(T=-1) == SHAPE and call(D=0) == SHAPE and call(stride=63) == SHAPE
    assert call(kind=2) == UNSUPPORTED
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert call(eps=eps) == UNSUPPORTED
    assert call(x=None) == NULL and call(w=None) == NULL and call(y=None) == NULL
    assert call(x=4097) == ALIGN and call(dt=1, x=4098) == ALIGN and call(res=4097) == ALIGN and call(w_dt=1, w=4098) == ALIGN
    assert call(mean=4098) == ALIGN and call(rstd=4098) == ALIGN and call(b=4097) == ALIGN and call(s=4097) == ALIGN
    assert call(T=0, x=None, w=None, y=None) == 0


def test_norm_backward_refuses(lib):
    f = lib.rlf_norm_bwd
    f.argtypes = [vp, i64, vp, i64, ci, i64, i32, vp, ci, ci, vp, vp, vp, vp, vp, vp, ci, vp, sz, vp]

    def call(dy=FAKE, dys=64, x=FAKE, xs=64, dt=0, T=4, D=64, w=FAKE, w_dt=0, kind=0, mean=None, rstd=FAKE, skip=None,
             gx=FAKE, gw=FAKE, gb=None, ws=FAKE, wsb=1 << 30):
        return f(dy, dys, x, xs, dt, T, D, w, w_dt, kind, mean, rstd, skip, gx, gw, gb, 0, ws, wsb, None)

    assert call(dt=3) == DTYPE and call(w_dt=9) == DTYPE and call(kind=-1) == UNSUPPORTED
    assert call(T=-1) == SHAPE and call(D=0) == SHAPE and call(dys=1) == SHAPE and call(xs=1) == SHAPE
    assert call(dy=None) == NULL and call(x=None) == NULL and call(w=None) == NULL and call(rstd=None) == NULL
    assert call(kind=1, mean=None) == NULL
    assert call(dy=4097) == ALIGN and call(skip=4097) == ALIGN and call(gx=4097) == ALIGN and call(gw=4098) == ALIGN
    assert call(rstd=4098) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=4100) == WORKSPACE and call(wsb=64) == WORKSPACE
    assert call(gw=None, gb=FAKE, ws=None) == WORKSPACE


def test_cross_entropy_refuses(lib):
    f = lib.rlf_cross_entropy_fwd_bwd
    f.argtypes = [vp, ci, i64, i32, i64, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, sz, vp, vp]

    def call(z=FAKE, dt=0, T=4, V=64, stride=64, ids=FAKE, mask=FAKE, eps=0.0, zc=0.0, denom=None, logp=FAKE, lse=None,
             loss=FAKE, grad=None, ws=FAKE, wsb=1 << 20):
        return f(z, dt, T, V, stride, ids, mask, eps, zc, denom, logp, lse, loss, grad, ws, wsb, None, None)

    assert call(dt=2) == DTYPE
    assert call(T=-1) == SHAPE and call(V=0) == SHAPE and call(stride=63) == SHAPE
    for eps in (-0.1, 1.1, float("nan")):
        assert call(eps=eps) == UNSUPPORTED
    for zc in (-1e-9, float("inf"), float("nan")):
        assert call(zc=zc) == UNSUPPORTED
    assert call(T=1 << 30, wsb=1 << 62) == UNSUPPORTED
    assert call(z=None) == NULL and call(ids=None) == NULL and call(logp=None) == NULL and call(loss=None) == NULL
    assert call(z=4097) == ALIGN and call(dt=1, z=4098) == ALIGN and call(grad=4097) == ALIGN and call(loss=4100) == ALIGN
    assert call(denom=4100) == ALIGN and call(lse=4098) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=4100) == WORKSPACE and call(wsb=256) == WORKSPACE


def test_fused_cross_entropy_refuses(lib):
    f = lib.rlf_fused_lmhead_cross_entropy
    f.argtypes = [vp, vp, i64, i32, i32, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, ci, ci, vp, sz, vp, vp]

    def call(H=FAKE, W=FAKE, T=4, D=64, V=64, ids=FAKE, eps=0.0, zc=0.0, denom=None, logp=FAKE, lse=None, loss=FAKE, gh=None,
             gw=None, gdt=1, acc=0, ws=FAKE, wsb=1 << 40):
        return f(H, W, T, D, V, ids, None, eps, zc, denom, logp, lse, loss, gh, gw, gdt, acc, ws, wsb, None, None)

    assert call(gdt=2) == DTYPE
    assert call(T=-1) == SHAPE and call(D=100) == SHAPE and call(V=63) == SHAPE and call(V=0) == SHAPE and call(D=0) == SHAPE
    assert call(eps=2.0) == UNSUPPORTED and call(zc=-1.0) == UNSUPPORTED and call(T=1 << 30) == UNSUPPORTED
    assert call(gw=FAKE, gdt=0, acc=1) == UNSUPPORTED
    assert call(H=None) == NULL and call(W=None) == NULL and call(ids=None) == NULL and call(logp=None) == NULL
    assert call(loss=None) == NULL
    assert call(H=4104) == ALIGN and call(W=4104) == ALIGN and call(gh=4104) == ALIGN and call(gw=4104) == ALIGN
    assert call(loss=4100) == ALIGN and call(denom=4100) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws=4100) == WORKSPACE and call(wsb=1000) == WORKSPACE


def test_workspace_sizes_grow_with_the_problem(lib):
    f = lib.rlf_workspace_bytes
    f.restype = sz
    f.argtypes = [ci, i64, i32, i32, ci]
    assert f(7, 0, 0, 64, 0) > 0 and f(7, 4096, 0, 64, 0) >= f(7, 64, 0, 64, 0) and f(7, 5, 0, 0, 0) == 0
    assert f(8, 0, 100, 0, 0) >= 256 and f(8, 1000, 100, 0, 0) >= 256 + 16000
    # the partial sums of long rows that a forward-only call streams; more of them for fp32 rows
    assert f(8, 1000, 151936, 0, 1) > f(8, 1000, 151936, 0, 0) > f(8, 1000, 100, 0, 0) and f(8, 1000, 0, 0, 0) == 0
    assert f(9, 100, 0, 64, 0) == 0
    # the scratch of a chunk, and an fp32 sum beside a bf16 gradient of more than one chunk
    assert f(9, 8192, 151936, 4096, 1) >= 2 * 8192 * 151936 and f(9, 18944, 512, 64, 0) == f(9, 18944, 512, 64, 1)
    assert f(9, 18945, 512, 64, 0) - f(9, 18945, 512, 64, 1) >= 4 * 512 * 64


def test_sizes_beyond_the_counters_are_refused(lib):
    """Columns, tokens and vocabulary entries are counted in 32 bits with room for one more step of a loop."""
    big = 1 << 30
    f = lib.rlf_norm_fwd
    f.argtypes = [vp, vp, ci, i64, i32, i64, vp, vp, ci, ci, f32, vp, vp, vp, vp, vp]
    for D in (big, 2 ** 31 - 1):
        assert f(FAKE, None, 0, 1, D, D, FAKE, None, 0, 0, 1e-6, None, FAKE, None, None, None) == UNSUPPORTED
    f = lib.rlf_norm_bwd
    f.argtypes = [vp, i64, vp, i64, ci, i64, i32, vp, ci, ci, vp, vp, vp, vp, vp, vp, ci, vp, sz, vp]
    assert f(FAKE, big, FAKE, big, 0, 1, big, FAKE, 0, 0, None, FAKE, None, FAKE, FAKE, None, 0, FAKE, 1 << 62, None) == UNSUPPORTED
    f = lib.rlf_cross_entropy_fwd_bwd
    f.argtypes = [vp, ci, i64, i32, i64, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    assert f(FAKE, 0, 1, big, big, FAKE, None, 0.0, 0.0, None, FAKE, None, FAKE, None, FAKE, 1 << 20, None, None) == UNSUPPORTED
    f = lib.rlf_fused_lmhead_cross_entropy
    f.argtypes = [vp, vp, i64, i32, i32, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, ci, ci, vp, sz, vp, vp]
    for D, V in ((64, big), (big, 64)):
        assert f(FAKE, FAKE, 1, D, V, FAKE, None, 0.0, 0.0, None, FAKE, None, FAKE, None, None, 1, 0, FAKE, 1 << 62, None,
                 None) == UNSUPPORTED
