"""Refusals of the attention's entry points, without a GPU: every bad size, type,
flag, stride, null or misaligned pointer is an error before any device work (none
is launched here)."""
import ctypes

import pytest
import torch

import paper_2511_21431_amd as mf
from paper_2511_21431_amd import _lib

INVALID, UNSUPPORTED = -1, -2
P = ctypes.c_void_p(4096)          # an aligned address that is never followed
ODD = ctypes.c_void_p(4096 + 8)
BYTE = ctypes.c_void_p(4096 + 2)
N = ctypes.c_void_p(0)
bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def attn(**kw):
    return mf.make_attn(**{**dict(heads=8, kv_heads=2, dim=64), **kw})


BAD = [(dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID),
       (dict(window=-1), INVALID), (dict(window=5, causal=False), INVALID), (dict(scale=0.0), INVALID),
       (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
       (dict(scale=float("inf")), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(dim=96, scale=1.0), UNSUPPORTED),
       (dict(dim=256), UNSUPPORTED), (dict(heads=2048), UNSUPPORTED)]


def fwd(a=None, T=4, seqs=1, off=P, Q=P, ldq=512, K=P, ldk=128, V=P, ldv=128, O=P, lse=P):
    a = attn() if a is None else a
    return _lib.lib().memfine_attn_fwd(T, seqs, ctypes.byref(a), off, Q, ldq, K, ldk, V, ldv, O, lse, None)


def bwd(a=None, T=4, seqs=1, off=P, Q=P, ldq=512, K=P, ldk=128, V=P, ldv=128, O=P, lse=P, dO=P,
        dQ=P, lddq=512, dK=P, lddk=128, dV=P, lddv=128):
    a = attn() if a is None else a
    return _lib.lib().memfine_attn_bwd(T, seqs, ctypes.byref(a), off, Q, ldq, K, ldk, V, ldv, O, lse, dO,
                                       dQ, lddq, dK, lddk, dV, lddv, None, None)


def test_packed_refusals():
    for kw, rc in BAD:
        assert fwd(attn(**kw)) == bwd(attn(**kw)) == rc, kw
    a = attn()
    a.causal = 2
    assert fwd(a) == bwd(a) == INVALID
    assert _lib.lib().memfine_attn_fwd(4, 1, None, P, P, 512, P, 128, P, 128, P, P, None) == INVALID
    for kw in (dict(T=-1), dict(seqs=-1), dict(ldq=504), dict(ldk=64), dict(ldv=132), dict(off=N),
               dict(Q=N), dict(K=N), dict(V=N), dict(O=N), dict(Q=ODD), dict(V=ODD), dict(O=ODD),
               dict(off=BYTE), dict(lse=BYTE)):
        assert fwd(**kw) == bwd(**kw) == INVALID, kw
    for kw in (dict(lse=N), dict(dO=N), dict(dQ=N), dict(dK=N), dict(dV=N), dict(dK=ODD), dict(lddq=64),
               dict(lddk=129), dict(lddv=120)):
        assert bwd(**kw) == INVALID, kw
    for kw in (dict(T=2 ** 31), dict(seqs=2 ** 20 + 1), dict(ldk=2 ** 20 + 8), dict(T=2 ** 31 - 1, seqs=1),
               dict(T=2 ** 24 + 1), dict(T=2 ** 20, seqs=2 ** 20)):
        assert fwd(**kw) == bwd(**kw) == UNSUPPORTED, kw
    # nothing to do
    for kw in (dict(T=0), dict(seqs=0)):
        assert fwd(off=N, Q=N, K=N, V=N, O=N, lse=N, **kw) == 0
        assert bwd(off=N, Q=N, dQ=N, **kw) == 0
    f = _lib.lib().memfine_attn_bwd_workspace_bytes
    alone = ctypes.byref(attn(kv_heads=8))              # no shared heads: two floats a row and head
    assert f(1000, 3, alone) == 2 * 1000 * 8 * 4 and f(0, 3, alone) == f(7, 0, alone) == 0
    assert f(1000, 1, ctypes.byref(attn())) >= 2 * 1000 * 8 * 4
    assert f(-1, 1, alone) < 0 and f(1, -1, alone) < 0 and f(1, 1, ctypes.byref(attn(heads=7))) < 0


def test_parts_of_the_gradient_follow_what_keys_are_seen_by():
    """Working memory of the gradient: none for partial sums where a short window leaves each
    block of keys few queries, as with no window where it is as long as the sequence, and
    never more with a window than without."""
    f = _lib.lib().memfine_attn_bwd_workspace_bytes

    def parts(T, seqs, **kw):
        a = attn(**kw)
        n = f(T, seqs, ctypes.byref(a)) - 2 * T * a.heads * 4
        each = 2 * T * a.kv_heads * a.dim * 4
        assert n % each == 0
        return n // each
    big = dict(heads=32, kv_heads=8, dim=128)
    assert parts(8192, 1, **big) == 2
    assert parts(8192, 1, window=128, **big) == parts(8192, 1, window=1024, **big) == 0
    assert parts(8192, 4, window=512, **big) == 0
    assert parts(4096, 1, causal=False, **big) == 2      # (all chains alike: two fill the device)
    for T, seqs, kw in ((8192, 1, big), (2048, 1, dict(heads=16, kv_heads=2)), (6783, 2, dict(heads=2)),
                        (900, 1, dict(heads=8, kv_heads=1, dtype=mf.F32))):
        kw = {**kw, "kv_heads": kw.get("kv_heads", kw["heads"])}
        whole = parts(T, seqs, **kw)
        assert all(parts(T, seqs, window=w, **kw) <= whole for w in (1, 64, 300, 1000, 2 ** 31 - 1))
        assert parts(T, seqs, window=T, **kw) == whole


def test_rope_refusals():
    def f(T=4, seqs=1, off=P, heads=3, dim=64, dtype=0, cos=P, sin=P, n=8, inter=0, inv=0, X=P, ldx=192,
          Y=P, ldy=192, null=False):
        r = _lib.Rotary(cos, sin, n, inter)
        return _lib.lib().memfine_rope(T, seqs, off, heads, dim, dtype, None if null else ctypes.byref(r),
                                       inv, X, ldx, Y, ldy, None)
    for kw in (dict(T=-1), dict(seqs=-2), dict(off=N), dict(heads=0), dict(dim=0), dict(cos=N), dict(sin=N),
               dict(sin=ODD), dict(n=0), dict(inter=2), dict(inv=-1), dict(X=N), dict(Y=N), dict(X=ODD),
               dict(ldx=128), dict(ldy=196), dict(ldy=200), dict(null=True), dict(off=BYTE)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(dim=32), dict(dtype=5), dict(heads=1025), dict(T=2 ** 31), dict(seqs=2 ** 21)):
        assert f(**kw) == UNSUPPORTED, kw
    assert f(T=0, off=N, X=N, Y=N) == f(seqs=0, off=N, X=N, Y=N) == 0


def cache(kv_heads=2, dim=64, page=16, pages=4, k=P, v=P, ks=N, vs=N):
    return _lib.Cache(kv_heads, dim, page, pages, k, v, ks, vs)


BAD_CACHE = [(dict(kv_heads=0), INVALID), (dict(page=8), INVALID), (dict(page=48), INVALID),
             (dict(pages=0), INVALID), (dict(k=N), INVALID), (dict(v=N), INVALID), (dict(ks=P), INVALID),
             (dict(vs=P), INVALID), (dict(k=ODD), INVALID), (dict(ks=ODD, vs=P), INVALID),
             (dict(page=2 ** 17), UNSUPPORTED), (dict(pages=2 ** 31), UNSUPPORTED),
             (dict(dim=80), UNSUPPORTED), (dict(page=65536, pages=1), 0)]


def test_write_refusals():
    def f(c=None, T=3, seqs=3, width=4, table=P, lengths=P, off=N, r=None, K=P, ldk=128, V=P, ldv=128,
          heads=8, Q=P, ldq=512, R=P):
        c = cache() if c is None else c
        return _lib.lib().memfine_kv_write(ctypes.byref(c), T, seqs, width, table, lengths, off,
                                           None if r is None else ctypes.byref(r), K, ldk, V, ldv, heads,
                                           Q, ldq, R, None)
    for kw, rc in BAD_CACHE:
        if rc:
            assert f(cache(**kw)) == rc, kw
    assert _lib.lib().memfine_kv_write(None, 3, 3, 4, P, P, N, None, P, 128, P, 128, 0, N, 0, N, None) == INVALID
    for kw in (dict(T=-1), dict(seqs=-1), dict(width=0), dict(T=4), dict(table=N), dict(lengths=N), dict(K=N),
               dict(V=N), dict(ldk=64), dict(ldv=130), dict(heads=-1), dict(heads=0), dict(Q=N), dict(R=N),
               dict(ldq=256), dict(Q=P, R=P, ldq=520), dict(K=ODD), dict(R=ODD), dict(table=BYTE),
               dict(lengths=BYTE), dict(off=BYTE), dict(r=_lib.Rotary(N, P, 4, 0)),
               dict(r=_lib.Rotary(P, P, 0, 0)), dict(r=_lib.Rotary(P, P, 4, 3))):
        assert f(**kw) == INVALID, kw
    for kw in (dict(width=2 ** 27), dict(heads=2000, ldq=2 ** 18), dict(T=2 ** 31, off=P),
               dict(seqs=2 ** 21, off=P)):
        assert f(**kw) == UNSUPPORTED, kw
    assert f(T=0, seqs=0, K=N, V=N, table=N) == 0


def test_decode_refusals():
    def f(a=None, c=None, seqs=3, width=4, table=P, lengths=P, Q=P, ldq=512, O=P, lse=P):
        a, c = attn() if a is None else a, cache() if c is None else c
        return _lib.lib().memfine_attn_decode(ctypes.byref(a), ctypes.byref(c), seqs, width, table, lengths,
                                              Q, ldq, O, lse, None, None)
    for kw, rc in BAD:
        assert f(attn(**kw)) == rc, kw
    for kw, rc in BAD_CACHE:
        if rc:
            assert f(c=cache(**kw)) == rc, kw
    assert f(attn(dtype=mf.F32)) == UNSUPPORTED
    for kw in (dict(a=attn(kv_heads=4)), dict(c=cache(dim=128)), dict(seqs=-1), dict(width=0), dict(table=N),
               dict(lengths=N), dict(Q=N), dict(O=N), dict(ldq=64), dict(Q=ODD), dict(O=ODD), dict(lse=BYTE),
               dict(table=BYTE)):
        assert f(**kw) == INVALID, kw
    assert f(width=2 ** 27) == UNSUPPORTED
    assert f(seqs=0, table=N, lengths=N, Q=N, O=N) == 0
    g = _lib.lib().memfine_attn_decode_workspace_bytes
    assert g(ctypes.byref(attn()), ctypes.byref(cache()), 0, 4) == 0
    assert g(ctypes.byref(attn()), ctypes.byref(cache()), 3, 4) > 0
    assert g(ctypes.byref(attn()), ctypes.byref(cache(page=24)), 3, 4) < 0


class Device:
    """A device tensor, as far as the binding looks."""
    is_cuda = True

    def __init__(self, *shape, dtype=bf, strides=None, device="cuda:0"):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)
        s = [1]
        for n in reversed(shape[1:]):
            s.insert(0, s[0] * n)
        self.strides, self.whole = strides or tuple(s), strides is None

    def is_contiguous(self):
        return self.whole

    def get_device(self):
        return self.device.index

    def stride(self):
        return self.strides

    def data_ptr(self):
        return 4096

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()


def test_binding_checks_shapes_types_and_strides():
    off = Device(2, dtype=i32)
    q, k = Device(5, 8, 64), Device(5, 2, 64)

    def call(**kw):
        a = {**dict(offsets=off, Q=q, K=k, V=k, O=q, lse=Device(8, 5, dtype=f32)), **kw}
        mf.memfine_attn_fwd(attn(), **a, stream=0)
    wide = (896, 64, 1)
    for kw, text in ((dict(Q=None), "Q is required"), (dict(offsets=None), "offsets is required"),
                     (dict(Q=Device(5, 7, 64)), "Q: shape"), (dict(K=Device(4, 2, 64)), "K: shape"),
                     (dict(V=Device(5, 2, 64, dtype=f32)), "V: dtype"),
                     (dict(K=Device(5, 2, 64, strides=(128, 1, 2))), "heads of a row"),
                     (dict(K=Device(5, 2, 64, strides=(256, 128, 1))), "heads of a row"),
                     (dict(O=Device(5, 8, 64, strides=wide)), "O must be contiguous"),
                     (dict(O=None), "O is required"), (dict(lse=Device(5, 8, dtype=f32)), "lse: shape"),
                     (dict(offsets=Device(2, dtype=torch.int64)), "offsets: dtype"),
                     (dict(K=Device(5, 2, 64, device="cuda:1")), "tensors on"),
                     (dict(Q=torch.zeros(5, 8, 64, dtype=bf)), "Q must be a device tensor")):
        with pytest.raises(ValueError, match=text):
            call(**kw)
    with pytest.raises(ValueError, match="lse is required"):
        mf.memfine_attn_bwd(attn(), off, q, k, k, q, None, q, q, k, k, stream=0)
    with pytest.raises(mf.MemfineError):     # rows 60 elements apart, then too few apart
        call(K=Device(5, 2, 64, strides=(132, 64, 1)))
    with pytest.raises(mf.MemfineError):
        call(K=Device(5, 2, 64, strides=(0, 64, 1)))
    page = Device(3, 2, 16, 64)
    c = mf.make_cache(page, page)
    for bad in (lambda: mf.make_cache(None, page), lambda: mf.make_cache(page, Device(3, 2, 16, 128)),
                lambda: mf.make_cache(page, page, Device(3, 2, 16, 2, dtype=u8)),
                lambda: mf.make_cache(Device(3, 2, 16, 64, dtype=u8), Device(3, 2, 16, 64, dtype=u8),
                                      Device(3, 2, 16, 2, dtype=u8)),
                lambda: mf.make_cache(torch.zeros(3, 2, 16, 64, dtype=bf), page)):
        with pytest.raises(ValueError):
            bad()
    table, n = Device(5, 4, dtype=i32), Device(5, dtype=i32)
    w = mf.memfine_kv_write
    for bad in (lambda: w(c, table, n, k, Device(5, 3, 64), stream=0), lambda: w(c, None, n, k, k, stream=0),
                lambda: w(c, table, Device(4, dtype=i32), k, k, stream=0),
                lambda: w(c, table, n, k, k, Q=q, stream=0),
                lambda: w(c, table, n, k, k, cos=Device(9, 32, dtype=f32), stream=0),
                lambda: w(c, table, n, k, k, cos=Device(9, 32, dtype=f32), sin=Device(8, 32, dtype=f32), stream=0),
                lambda: w(c, table, n, k, k, offsets=Device(5, dtype=i32), stream=0),
                lambda: mf.memfine_attn_decode(attn(), c, table, n, Device(4, 8, 64), q, stream=0),
                lambda: mf.memfine_attn_decode(attn(), c, table, n, q, None, stream=0),
                lambda: mf.memfine_rope(off, Device(9, 32, dtype=f32), Device(9, 31, dtype=f32), q, q, stream=0),
                lambda: mf.memfine_rope(off, Device(9, 32, dtype=f32), Device(9, 32, dtype=f32), q, k, stream=0)):
        with pytest.raises(ValueError):
            bad()
