"""GPU parity of the MX4 matrices (layout, rounding, values), of the linear map
and of the expert layer's forward with MX4 weights, against oracle/around.py
in float64 on the same held values.

Tolerances, from the arithmetic (u = 2^-24):
* layout, codes and scales: exact; values exact.
* linear, bf16 activations: products are exact in fp32; sums of at most K / 8 +
  64 steps: (K / 8 + 64) u of sum |x w|; MX8: and 2^-14 of the largest product of
  each 128 (how the matrix core aligns them).  bf16 output: 2^-8 more.
* experts: a (rounded to bf16) and Y (rounded to bf16) have independent errors
  of at most 2^-8 / sqrt(3) rms each: 4e-3 of the 2-norm, and 2e-2 of the largest |Y|
  (the layer's own tolerance) per element.  On MX8 a value of a next to a
  rounding boundary may go to the other side (one part in sixteen of one of the
  F terms): 5e-3 of the 2-norm and 5e-2 per element, F >= 256.
"""
import numpy as np
import pytest

from gpu_harness import torch
from oracle import around as oa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    t = torch()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_21431_amd as m
    m.lib()
    return m


def dev(a, dtype=None):
    x = torch().from_numpy(np.ascontiguousarray(a)).cuda()
    return x if dtype is None else x.to(dtype)


def f64(x):
    return x.detach().cpu().double().numpy()


def rows(rng, E, N, K, lo=118, hi=124):
    """Row-major MX4 codes, scales and their values."""
    code = rng.integers(0, 16, (E, N, K)).astype(np.uint8)
    s = rng.integers(lo, hi, (E, N, K // 32)).astype(np.uint8)
    v = np.where(code >= 8, -1.0, 1.0) * oa.E2M1[code & 7]
    return oa.mx4_row_codes(code), s, v * np.repeat(2.0 ** (s - 127.0), 32, axis=2)


def packed(mf, E, N, K, c, s):
    return mf.memfine_mxw_pack(E, N, K, dev(c), dev(s))


def activations(rng, T, K, mx8, std=1.0):
    """(X, XS) on the device and their values."""
    t = torch()
    x = rng.standard_normal((T, K)) * std
    if not mx8:
        X = t.from_numpy(x).to(t.bfloat16)
        return X.cuda(), None, f64(X)
    code, s, v = oa.mx_round(x, "mx8")
    return dev(code), dev(s), v


SHAPES = [(1, 16, 32), (2, 48, 160), (1, 64, 512), (3, 32, 544), (1, 272, 1056)]


@pytest.mark.parametrize("E,N,K", SHAPES)
def test_pack_and_unpack(mf, E, N, K):
    t = torch()
    rng = np.random.default_rng(N + K)
    c, s, v = rows(rng, E, N, K, 0, 255)
    codes, scales = packed(mf, E, N, K, c, s)
    wc, ws = oa.mx4_layout(c, s)
    assert np.array_equal(codes.cpu().numpy(), wc) and np.array_equal(scales.cpu().numpy(), ws)
    W = t.full((E, N, K), float("nan"), device="cuda")
    mf.memfine_mxw_unpack(codes, scales, W)
    with np.errstate(over="ignore"):
        assert np.array_equal(f64(W), v.astype(np.float32).astype(np.float64))
    s = rng.integers(100, 150, s.shape).astype(np.uint8)
    mf.memfine_mxw_pack(E, N, K, dev(c), dev(s), codes, scales)
    B = t.full((E, N, K), float("nan"), dtype=t.bfloat16, device="cuda")
    mf.memfine_mxw_unpack(codes, scales, B)
    v = np.where(np.signbit(v), -1.0, 1.0) * np.abs(np.where(c_values(c) == 0, 0, c_values(c)))
    assert np.array_equal(f64(B), v * np.repeat(2.0 ** (s - 127.0), 32, axis=2))


def c_values(c):
    code = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
    return np.where(code >= 8, -1.0, 1.0) * oa.E2M1[code & 7]


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("E,N,K", SHAPES)
def test_quantize(mf, E, N, K, dtype):
    t = torch()
    rng = np.random.default_rng(N * K)
    x = rng.standard_normal((E, N, K)) * 2.0 ** rng.integers(-20, 20, (E, N, 1))
    x[0, 0, :32] = 0
    x[0, 1, :32] = np.linspace(-6, 6, 32)
    x[0, 2, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]     # ties
    x[0, 2, 8:32] = 0
    W = t.from_numpy(x).to(t.bfloat16 if dtype == "bf16" else t.float32).cuda()
    codes, scales = mf.memfine_mxw_quantize(W)
    code, s, v = oa.mx_round(f64(W), "mx4")
    wc, ws = oa.mx4_layout(oa.mx4_row_codes(code), s)
    assert np.array_equal(scales.cpu().numpy(), ws)
    assert np.array_equal(codes.cpu().numpy(), wc)


def test_quantize_marks_blocks_that_are_not_finite(mf):
    t = torch()
    W = t.ones((1, 16, 96))
    W[0, 3, 40] = float("nan")
    W[0, 4, 0] = float("-inf")
    codes, scales = mf.memfine_mxw_quantize(W.cuda())
    V = t.zeros((1, 16, 96), device="cuda")
    mf.memfine_mxw_unpack(codes, scales, V)
    bad = t.zeros((16, 96), dtype=t.bool)
    bad[3, 32:64] = True
    bad[4, :32] = True
    assert t.equal(t.isnan(V[0].cpu()), bad) and t.all(V[0].cpu()[~bad] == 1)


LINEAR = [(1, 16, 32), (1, 4096, 7168), (2, 48, 160), (15, 272, 544), (16, 512, 1024),
          (17, 208, 2080), (33, 1008, 96), (48, 576, 4096), (100, 320, 1408), (257, 528, 736),
          (600, 1024, 512)]


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,N,K", LINEAR)
def test_linear(mf, T, N, K, mx8):
    t = torch()
    rng = np.random.default_rng(T + N + K)
    c, s, W = rows(rng, 1, N, K)
    codes, scales = packed(mf, 1, N, K, c, s)
    X, XS, x = activations(rng, T, K, mx8)
    ref, mag = x @ W[0].T, np.abs(x) @ np.abs(W[0]).T
    tol = (K / 8 + 64) * 2.0 ** -24 * mag
    if mx8:
        pad = -K % 128
        xa = np.pad(np.abs(x), ((0, 0), (0, pad))).reshape(T, -1, 128).max(axis=2)
        wa = np.pad(np.abs(W[0]), ((0, 0), (0, pad))).reshape(N, -1, 128).max(axis=2)
        tol = tol + 2.0 ** -14 * (xa @ wa.T)
    for dt in (t.float32, t.bfloat16):
        out = t.full((T + 20, N), float("nan"), dtype=dt, device="cuda")
        out[T:] = 7
        mf.memfine_linear_mxw(N, K, X, codes, scales, out[:T], XS=XS)
        half = 2.0 ** -8 if dt == t.bfloat16 else 0.0
        assert np.all(np.abs(f64(out[:T]) - ref) <= tol + half * (np.abs(ref) + tol))
        assert t.all(out[T:] == 7)


@pytest.mark.parametrize("T", (3, 40, 200))
def test_linear_keeps_rows_apart(mf, T):
    """A row that is not finite stays so and leaves the others; K off the tile
    multiplies nothing past the row's end."""
    t = torch()
    rng = np.random.default_rng(T)
    N, K = 96, 160
    c, s, W = rows(rng, 1, N, K)
    codes, scales = packed(mf, 1, N, K, c, s)
    for mx8 in (False, True):
        X, XS, x = activations(rng, T, K, mx8)
        clean = t.zeros((T, N), device="cuda")
        mf.memfine_linear_mxw(N, K, X, codes, scales, clean, XS=XS)
        # the rows lie between NaNs in memory
        if mx8:
            big, bs = t.full((T + 2, K), 0x7f, dtype=t.uint8).cuda(), t.full((T + 2, K // 32), 255, dtype=t.uint8).cuda()
            bs[1:-1] = XS
            XS = bs[1:-1]
            assert XS.is_contiguous()
        else:
            big = t.full((T + 2, K), float("nan"), dtype=t.bfloat16, device="cuda")
        big[1:-1] = X
        Y = t.zeros((T, N), device="cuda")
        mf.memfine_linear_mxw(N, K, big[1:-1], codes, scales, Y, XS=XS)
        assert t.equal(Y, clean)
        if mx8:
            XS[T // 2, 1] = 255
        else:
            big[1 + T // 2, 50] = float("nan")
        mf.memfine_linear_mxw(N, K, big[1:-1], codes, scales, Y, XS=XS)
        keep = t.arange(T) != T // 2
        assert t.all(t.isnan(Y[T // 2])) and t.equal(Y[keep], clean[keep])


def test_linear_scales_over_their_range(mf):
    """Scale bytes from the smallest normal results to the largest."""
    t = torch()
    rng = np.random.default_rng(1)
    N, K = 32, 256
    for mx8 in (False, True):
        for ws in (30, 127, 200):
            c, s, W = rows(rng, 1, N, K, ws, ws + 8)
            codes, scales = packed(mf, 1, N, K, c, s)
            X, XS, x = activations(rng, 5, K, mx8)
            Y = t.zeros((5, N), device="cuda")
            mf.memfine_linear_mxw(N, K, X, codes, scales, Y, XS=XS)
            ref, mag = x @ W[0].T, np.abs(x) @ np.abs(W[0]).T
            assert np.all(np.abs(f64(Y) - ref) <= 2.0 ** -12 * mag)


# ----------------------------------------------------------------- experts
def experts_case(rng, T, h, F, E, k, mx8, idx=None):
    c1, s1, W1 = rows(rng, E, 2 * F, h, 119, 122)
    c2, s2, W2 = rows(rng, E, h, F, 119, 122)
    X, XS, x = activations(rng, T, h, mx8, 16 / np.sqrt(h))
    if idx is None:
        idx = rng.integers(0, E, (T, k))
    g = rng.random((T, k)).astype(np.float32)
    return (c1, s1, W1), (c2, s2, W2), X, XS, x, np.asarray(idx, dtype=np.int32), g


def run_experts(mf, T, h, F, E, k, mats, X, XS, idx, g, chunks=1, **kw):
    t = torch()
    (c1, s1, _), (c2, s2, _) = mats
    p1, p2 = packed(mf, E, 2 * F, h, c1, s1), packed(mf, E, h, F, c2, s2)
    Y = t.full((T, h), float("nan"), dtype=t.bfloat16, device="cuda")
    mf.memfine_moe_fwd_mxw(mf.make_shape(T, h, F, E, k, mf.BF16), chunks, X, dev(idx), dev(g), *p1,
                           *p2, Y, XS=XS, **kw)
    return Y


def check(Y, ref, mx8):
    got = f64(Y)
    assert np.all(np.isfinite(got))
    err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    worst = np.max(np.abs(got - ref)) / np.max(np.abs(ref))
    assert err <= (5e-3 if mx8 else 4e-3) and worst <= (5e-2 if mx8 else 2e-2), (err, worst)


EXPERTS = [  # T, h, F, E, k
    (1, 64, 256, 1, 1), (1, 512, 256, 8, 3), (2, 576, 320, 5, 2), (5, 128, 256, 40, 8),
    (16, 256, 256, 4, 4), (33, 320, 448, 70, 2), (64, 512, 256, 3, 2), (200, 256, 320, 2, 1),
    (300, 448, 256, 6, 4), (700, 128, 256, 16, 6), (1000, 192, 256, 3, 5)]


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,h,F,E,k", EXPERTS)
def test_experts(mf, T, h, F, E, k, mx8):
    rng = np.random.default_rng(T * 7 + h)
    m1, m2, X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, mx8)
    ref = oa.moe_fwd_mx(x, idx, g, m1[2], m2[2], mx8)
    Y = run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g)
    check(Y, ref, mx8)
    t = torch()
    assert t.equal(run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g), Y)
    for chunks in (2, 5):
        check(run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g, chunks=chunks), ref, mx8)


@pytest.mark.parametrize("mx8", (False, True))
def test_experts_uneven_loads_and_dropped_slots(mf, mx8):
    """One expert takes nearly all, others one row or none; ids outside [0, E)
    add nothing; a token whose slots are all dropped gets zeros."""
    rng = np.random.default_rng(3)
    T, h, F, E, k = 150, 256, 256, 12, 3
    idx = np.full((T, k), 7)
    idx[5, 1], idx[9, 0], idx[149, 2] = 0, 11, 3
    idx[20], idx[40, 1], idx[0, 0] = -1, E, 1 << 30
    m1, m2, X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, mx8, idx)
    Y = run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g)
    ok = (idx >= 0) & (idx < E)
    ref = oa.moe_fwd_mx(x, np.where(ok, idx, 0), np.where(ok, g, 0), m1[2], m2[2], mx8)
    check(Y, ref, mx8)
    assert torch().all(Y[20] == 0)
    one = np.full((1, 2), -1)
    m1, m2, X, XS, x, idx, g = experts_case(rng, 1, h, F, E, 2, mx8, one)
    assert torch().all(run_experts(mf, 1, h, F, E, 2, (m1, m2), X, XS, idx, g) == 0)


def test_experts_memory_and_streams(mf):
    """The caller's allocator serves the documented bytes; a failing one is an
    error that leaves nothing allocated; a call on a side stream waits for that
    stream's work."""
    t = torch()
    rng = np.random.default_rng(4)
    T, h, F, E, k = 60, 256, 256, 6, 2
    for mx8 in (False, True):
        m1, m2, X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, mx8)
        ref = run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g)
        shape = mf.make_shape(T, h, F, E, k, mf.BF16)
        for chunks in (1, 3):
            a = mf.TorchAllocator()
            run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g, chunks=chunks, allocator=a)
            assert a.high_water == mf.memfine_moe_mxw_workspace_bytes(shape, chunks, mx8)
            assert a.live_bytes == 0
        a = mf.TorchAllocator()
        a.fail_at = 1
        with pytest.raises(mf.MemfineError) as e:
            run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g, allocator=a)
        assert e.value.code == -4 and a.live_bytes == 0
        side = t.cuda.Stream()
        late = t.zeros_like(X)
        t.cuda.synchronize()
        with t.cuda.stream(side):
            for _ in range(50):
                late.copy_(X)
            Y = run_experts(mf, T, h, F, E, k, (m1, m2), late, XS, idx, g)
        side.synchronize()
        assert t.equal(Y, ref)


def test_experts_agree_with_the_bf16_layer(mf):
    """On weights that bf16 holds exactly (every MX4 value), the bf16 layer
    computes the same map."""
    t = torch()
    rng = np.random.default_rng(6)
    T, h, F, E, k = 96, 256, 256, 4, 2
    m1, m2, X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, False)
    Y = run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g)
    Z = t.zeros_like(Y)
    mf.memfine_moe_fwd(mf.make_shape(T, h, F, E, k, mf.BF16), 1, X, dev(idx), dev(g),
                       dev(m1[2], t.bfloat16), dev(m2[2], t.bfloat16), Z)
    assert np.linalg.norm(f64(Y) - f64(Z)) <= 8e-3 * np.linalg.norm(f64(Z))
