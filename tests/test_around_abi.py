"""Refusals of the entry points around the layer, without a GPU: every bad
size, type, flag, null or misaligned pointer is an error before any device
work (none is launched here)."""
import ctypes

import pytest
import torch

import paper_2511_21431_amd as mf
from paper_2511_21431_amd import _lib

INVALID, UNSUPPORTED = -1, -2
P = ctypes.c_void_p(4096)          # an aligned address that is never followed
ODD = ctypes.c_void_p(4096 + 8)
N = ctypes.c_void_p(0)


def fwd(T=4, h=64, dtype=0, eps=1e-6, X=P, R=N, w=P, S=N, Y=P, Q=N, QS=N):
    return _lib.lib().memfine_norm_fwd(T, h, dtype, eps, X, R, w, S, Y, Q, QS, None)


def test_norm_refusals():
    for kw in (dict(T=-1), dict(h=0), dict(h=96), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(X=N), dict(w=N), dict(Y=N), dict(S=P), dict(Q=P),
               dict(QS=P), dict(X=ODD), dict(w=ODD), dict(Y=ODD), dict(R=ODD),
               dict(R=P, S=ODD)):
        assert fwd(**kw) == INVALID, kw
    for kw in (dict(dtype=2), dict(h=16384 + 64), dict(T=2**31)):
        assert fwd(**kw) == UNSUPPORTED, kw
    assert fwd(T=0, X=N, w=N, Y=N) == 0

    def bwd(T=4, h=64, dtype=1, eps=0.0, X=P, w=P, dY=P, dS=N, dX=P, dw=P, acc=0):
        return _lib.lib().memfine_norm_bwd(T, h, dtype, eps, X, w, dY, dS, dX, dw, acc, None, None)
    for kw in (dict(T=-1), dict(h=32), dict(X=N), dict(w=N), dict(dY=N), dict(dX=N), dict(dw=N),
               dict(acc=2), dict(dS=ODD), dict(dw=ODD)):
        assert bwd(**kw) == INVALID, kw
    assert bwd(dtype=3) == UNSUPPORTED
    assert bwd(T=0, acc=1) == 0


def test_mx_values_refusals():
    f = _lib.lib().memfine_mx_values
    assert f(-1, 64, P, P, 0, P, None) == INVALID
    assert f(1, 48, P, P, 0, P, None) == INVALID
    assert f(1, 64, N, P, 0, P, None) == INVALID
    assert f(1, 64, P, P, 0, ODD, None) == INVALID
    assert f(1, 64, P, P, 5, P, None) == UNSUPPORTED
    assert f(0, 64, N, N, 0, N, None) == 0


def test_route_refusals():
    L = _lib.lib()
    good = dict(E=64, k=6, score="sigmoid", groups=8, top_groups=2)

    def both(T=3, z=P, b=N, i=P, g=P, d=P, **kw):
        a = ctypes.byref(mf.make_gating(**{**good, **kw}))
        return (L.memfine_route_fwd(T, a, z, b, i, g, None),
                L.memfine_route_bwd(T, a, z, i, g, d, None))
    for kw in (dict(T=-1), dict(E=0, k=0), dict(k=0), dict(k=65), dict(groups=0),
               dict(groups=7), dict(top_groups=0), dict(top_groups=9), dict(k=9, top_groups=1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(z=N), dict(i=N),
               dict(z=ODD), dict(i=ODD)):
        assert both(**kw) == (INVALID, INVALID), kw
    assert both(b=ODD)[0] == INVALID and both(d=N)[1] == INVALID
    for kw in (dict(E=512), dict(k=17, top_groups=8), dict(groups=32, top_groups=32),
               dict(T=2**31)):
        assert both(**kw) == (UNSUPPORTED, UNSUPPORTED), kw
    assert both(T=0, z=N, i=N, g=N, d=N) == (0, 0)
    assert L.memfine_route_fwd(1, None, P, N, P, P, None) == INVALID
    bad = mf.make_gating(**good)
    bad.score = 2
    assert L.memfine_route_fwd(1, ctypes.byref(bad), P, N, P, P, None) == INVALID
    bad = mf.make_gating(**good)
    bad.renorm = 2
    assert L.memfine_route_bwd(1, ctypes.byref(bad), P, P, P, P, None) == INVALID
    with pytest.raises(ValueError):
        mf.make_gating(8, 2, score="tanh")


def test_router_logits_refusals():
    L = _lib.lib()
    s = lambda **kw: ctypes.byref(mf.make_shape(**{**dict(T=4, h=64, F=64, E=8, k=2, dtype=0), **kw}))  # noqa: E731
    assert L.memfine_router_logits(s(E=257), P, P, P, None) == UNSUPPORTED
    assert L.memfine_router_logits(s(h=65), P, P, P, None) == INVALID
    assert L.memfine_router_logits(s(), N, P, P, None) == INVALID
    assert L.memfine_router_logits(s(), P, ODD, P, None) == INVALID
    assert L.memfine_router_logits(s(T=0), N, N, N, None) == 0
    b = L.memfine_router_logits_bwd
    assert b(s(E=257), P, P, P, P, P, 0, 0, None, None) == UNSUPPORTED
    assert b(s(), P, P, P, P, P, 2, 0, None, None) == INVALID
    assert b(s(), P, P, N, P, P, 0, 0, None, None) == INVALID
    assert b(s(), P, N, P, P, P, 0, 0, None, None) == INVALID
    assert b(s(), P, P, P, ODD, P, 0, 0, None, None) == INVALID


def test_mxw_refusals():
    L = _lib.lib()
    assert mf.memfine_mxw_code_bytes(16, 32) == 1024
    assert mf.memfine_mxw_code_bytes(48, 160) == 3 * 2 * 1024
    assert mf.memfine_mxw_scale_bytes(48, 160) == 3 * 256
    assert mf.memfine_mxw_scale_bytes(16, 544) == 2 * 256
    for n, k in ((0, 32), (8, 32), (24, 32), (16, 0), (16, 48)):
        assert L.memfine_mxw_code_bytes(n, k) < 0 and L.memfine_mxw_scale_bytes(n, k) < 0
        assert L.memfine_mxw_pack(1, n, k, P, P, P, P, None) == INVALID
        assert L.memfine_mxw_quantize(1, n, k, 0, P, P, P, None) == INVALID
        assert L.memfine_mxw_unpack(1, n, k, P, P, 0, P, None) == INVALID
        assert L.memfine_linear_mxw(1, n, k, P, N, P, P, 0, P, None) == INVALID
    assert L.memfine_mxw_pack(0, 16, 32, P, P, P, P, None) == INVALID
    assert L.memfine_mxw_pack(1, 16, 32, N, P, P, P, None) == INVALID
    assert L.memfine_mxw_pack(1, 16, 32, ODD, P, P, P, None) == INVALID
    assert L.memfine_mxw_quantize(1, 16, 32, 2, P, P, P, None) == UNSUPPORTED
    assert L.memfine_mxw_quantize(1, 16, 32, 0, P, P, N, None) == INVALID
    assert L.memfine_mxw_unpack(1, 16, 32, P, P, 2, P, None) == UNSUPPORTED
    assert L.memfine_mxw_unpack(1, 16, 32, P, P, 0, ODD, None) == INVALID
    f = lambda T=1, X=P, XS=N, c=P, s=P, d=0, Y=P: L.memfine_linear_mxw(T, 16, 32, X, XS, c, s, d, Y, None)  # noqa: E731
    for kw in (dict(T=-1), dict(X=N), dict(c=N), dict(s=N), dict(Y=N), dict(X=ODD), dict(Y=ODD)):
        assert f(**kw) == INVALID, kw
    assert f(d=2) == UNSUPPORTED and f(T=2**31) == UNSUPPORTED
    assert f(T=0, X=N, Y=N) == 0


def test_moe_mxw_refusals():
    L = _lib.lib()

    def f(X=P, XS=N, idx=P, g=P, c1=P, s1=P, c2=P, s2=P, Y=P, chunks=1, **kw):
        s = mf.make_shape(**{**dict(T=4, h=64, F=64, E=8, k=2, dtype=0), **kw})
        return L.memfine_moe_fwd_mxw(ctypes.byref(s), chunks, X, XS, idx, g, c1, s1, c2, s2, Y,
                                     None, None)
    for kw in (dict(X=N), dict(idx=N), dict(g=N), dict(c1=N), dict(s1=N), dict(c2=N), dict(s2=N),
               dict(Y=N), dict(chunks=0), dict(T=-1), dict(h=96), dict(F=32), dict(E=0),
               dict(X=ODD), dict(c2=ODD), dict(Y=ODD)):
        assert f(**kw) == INVALID, kw
    assert f(dtype=1) == UNSUPPORTED
    assert f(T=0, X=N) == 0
    s = mf.make_shape(100, 64, 128, 8, 2, mf.BF16)
    assert mf.memfine_moe_mxw_workspace_bytes(s, 1) > mf.memfine_moe_mxw_workspace_bytes(s, 4)
    assert mf.memfine_moe_mxw_workspace_bytes(s, 1) > mf.memfine_moe_mxw_workspace_bytes(s, 1, True)
    assert mf.memfine_moe_mxw_workspace_bytes(mf.make_shape(0, 64, 128, 8, 2, mf.BF16), 1) == 0
    with pytest.raises(mf.MemfineError):
        mf.memfine_moe_mxw_workspace_bytes(mf.make_shape(100, 64, 128, 8, 2, mf.F32), 1)
    with pytest.raises(mf.MemfineError):
        mf.memfine_moe_mxw_workspace_bytes(s, 0)


def test_binding_checks_shapes_types_and_strides():
    """The binding refuses what the C call could not see: shapes, dtypes,
    strides, host tensors."""
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    X, w = torch.zeros(4, 64, dtype=bf), torch.zeros(64, dtype=bf)
    Y = torch.zeros(4, 64, dtype=bf)
    bad = [
        lambda: mf.memfine_norm_fwd(1e-6, X, w, Y=Y),                          # host tensors
        lambda: mf.memfine_norm_fwd(1e-6, X.half(), w, Y=Y),
        lambda: mf.memfine_norm_fwd(1e-6, X[0], w, Y=Y),
        lambda: mf.memfine_norm_fwd(1e-6, None, w, Y=Y),
        lambda: mf.memfine_norm_fwd(1e-6, torch.zeros(64, 4, dtype=bf).t(), w, Y=Y),
        lambda: mf.memfine_mx_values(torch.zeros(4, 64, dtype=u8), torch.zeros(4, 3, dtype=u8), Y),
        lambda: mf.memfine_route_fwd(mf.make_gating(8, 2), torch.zeros(4, 9), None, None),
        lambda: mf.memfine_linear_mxw(16, 64, X.float(), torch.zeros(1, 1024, dtype=u8),
                                      torch.zeros(1, 256, dtype=u8), Y),
        lambda: mf.memfine_linear_mxw(16, 64, X, torch.zeros(1, 1000, dtype=u8),
                                      torch.zeros(1, 256, dtype=u8), Y),
        lambda: mf.memfine_mxw_quantize(torch.zeros(1, 20, 64, dtype=bf)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, mf.MemfineError)):
            f()
