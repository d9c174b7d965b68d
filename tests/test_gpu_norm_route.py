"""GPU parity of the residual RMS norm and of routing from logits against
oracle/around.py, which starts from the same stored inputs in float64.

Tolerances, from the arithmetic (u = 2^-24, the fp32 unit; every sum in fp32):
* S: the fp32 sum of two stored values rounded once: bit-exact.
* Y: the mean of squares is a chain of at most 8 products a lane, 6 + 16 steps
  over lanes and waves, halved by the root, and four more roundings: below 32 u
  = 2e-6 of |Y|; plus half a unit of bf16, 2^-8.
* MX8 of Y: within half a step of e4m3 (2^-4 of the value, 2^-10 of the scale
  below the normals) of Y, with the scale of Y's own block unless the block's
  maximum lies within 1e-5 of the scale's limit.
* dX: the two row sums as above: 2^-8 (bf16) + 1e-5 of the sum of the
  magnitudes of its three terms.
* dw: T rows in at most T + 20 steps: (T + 20) u + 2e-6 of the sum of magnitudes.
* gates: e^x to 2 u, sums of at most 16 + 4 terms, a reciprocal and products:
  below 40 u, 4e-6 with margin; dlogits 1e-5 of the sum of the magnitudes of
  their terms (differences of gates appear in it).
* idx: equal, on logits whose selection no rounding can change, or exact ties.
"""
import itertools

import numpy as np
import pytest

from gpu_harness import torch
from oracle import around as oa
from oracle import router as orr

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def mf():
    t = torch()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_21431_amd as m
    m.lib()
    return m


def gen(seed):
    return torch().Generator().manual_seed(seed)


def draw(g, *shape, dtype="f32", std=1.0):
    t = torch()
    x = t.randn(*shape, generator=g) * std
    return x.to(t.bfloat16 if dtype == "bf16" else t.float32)


def f64(x):
    return x.detach().cpu().double().numpy()


def nan_out(shape, like):
    return torch().full(shape, float("nan"), dtype=like.dtype, device="cuda")


SIZES = [(1, 64), (2, 512), (3, 576), (17, 1088), (5, 4096), (33, 7168), (2, 16384)]


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,h", SIZES)
def test_norm_forward(mf, T, h, dtype):
    t = torch()
    g = gen(T * 7919 + h)
    X, R, w = draw(g, T, h, dtype=dtype), draw(g, T, h, dtype=dtype, std=3), draw(g, h, dtype=dtype)
    X[0, :32] = 0
    R[0, :32] = 0                       # a block of zeros
    X[-1] *= 1e-3
    Xd, Rd, wd = X.cuda(), R.cuda(), w.cuda()
    S, Y = nan_out((T, h), X), nan_out((T, h), X)
    Q = t.full((T, h), 0x7f, dtype=t.uint8, device="cuda")
    QS = t.full((T, h // 32), 9, dtype=t.uint8, device="cuda")
    V = nan_out((T, h), X)
    mf.memfine_norm_fwd(EPS, Xd, wd, R=Rd, S=S, Y=Y, Q=Q, QS=QS)
    mf.memfine_mx_values(Q, QS, V)
    want_S = (X.float() + R.float()).to(X.dtype)
    assert t.equal(S.cpu(), want_S)
    ref = oa.norm_fwd(f64(want_S), f64(w), EPS)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert np.all(np.abs(f64(Y) - ref) <= (half + 2e-6) * np.abs(ref) + 1e-38)
    top = np.abs(ref).reshape(T, -1, 32).max(axis=2)
    s = QS.cpu().numpy().astype(np.float64)
    lim = 448 * 2.0 ** (s - 127)
    assert np.all((top <= lim * (1 + 1e-5)) & ((top > lim / 2 * (1 - 1e-5)) | (s == 0)))
    scale = np.repeat(2.0 ** (s - 127), 32, axis=1)
    assert np.all(np.abs(f64(V) - ref) <= (1 + 1e-4) * np.maximum(np.abs(ref) * 2.0 ** -4,
                                                                  scale * 2.0 ** -10) + 1e-38)
    # the same without the residual, S, MX8; and in place
    Y2 = nan_out((T, h), X)
    mf.memfine_norm_fwd(EPS, S, wd, Y=Y2)
    assert t.equal(Y2, Y)
    mf.memfine_norm_fwd(EPS, Xd, wd, R=Rd, S=Rd, Q=Q, QS=QS)
    assert t.equal(Rd, S)


def test_norm_rows_that_are_not_finite_or_zero(mf):
    """A row of zeros is zeros, a NaN or infinity stays in its row; in MX8 it
    makes its blocks NaN."""
    t = torch()
    h = 512
    X = t.randn(5, h, generator=gen(3)).to(t.bfloat16)
    X[1] = 0
    X[2, 100] = float("nan")
    X[3, 7] = float("inf")
    w = t.ones(h, dtype=t.bfloat16)
    Y = nan_out((5, h), X)
    Q = t.zeros((5, h), dtype=t.uint8, device="cuda")
    QS = t.zeros((5, h // 32), dtype=t.uint8, device="cuda")
    V = nan_out((5, h), X)
    mf.memfine_norm_fwd(EPS, X.cuda(), w.cuda(), Y=Y, Q=Q, QS=QS)
    mf.memfine_mx_values(Q, QS, V)
    Y, V, QS = Y.cpu(), V.cpu(), QS.cpu()
    assert t.all(Y[1] == 0) and t.all(V[1] == 0)
    assert t.all(t.isnan(Y[2])) and t.all(t.isnan(V[2])) and t.all(QS[2] == 255)
    assert t.isnan(Y[3, 7]) and t.all(Y[3, :7] == 0) and t.all(t.isnan(V[3, :32]))
    assert t.all(V[3, 32:] == 0)
    assert t.all(t.isfinite(Y[[0, 1, 4]].float())) and t.all(t.isfinite(V[[0, 1, 4]].float()))


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,h,residual", [(1, 64, True), (3, 576, False), (700, 512, True),
                                          (33, 7168, True), (2100, 1088, False), (2, 16384, True)])
def test_norm_backward(mf, T, h, residual, dtype):
    t = torch()
    g = gen(T * 31 + h)
    X, w, dY, dS = (draw(g, *s, dtype=dtype) for s in ((T, h), (h,), (T, h), (T, h)))
    dS = dS if residual else None
    dev = [None if a is None else a.cuda() for a in (X, w, dY, dS)]
    dX = nan_out((T, h), X)
    dw = t.full((h,), float("nan"), device="cuda")
    mf.memfine_norm_bwd(EPS, dev[0], dev[1], dev[2], dX, dw, dS=dev[3])
    x, ww, dy = f64(X), f64(w), f64(dY)
    rX, rw = oa.norm_bwd(x, ww, dy, None if dS is None else f64(dS), EPS)
    r = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + EPS)
    mag = r * (np.abs(dy * ww) + np.abs(x) * r * r * np.abs(dy * ww * x).mean(axis=1, keepdims=True))
    mag = mag + (0 if dS is None else np.abs(f64(dS)))
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert np.all(np.abs(f64(dX) - rX) <= (half + 1e-5) * mag)
    mag_w = np.abs(dy * x * r).sum(axis=0)
    tol_w = ((T + 20) * 2.0 ** -24 + 2e-6) * mag_w
    assert np.all(np.abs(f64(dw) - rw) <= tol_w)
    # accumulation, in place of dY, repeatable bit for bit
    acc = dw.clone()
    mf.memfine_norm_bwd(EPS, dev[0], dev[1], dev[2], dev[2], acc, dS=dev[3], accumulate_dw=True)
    assert t.equal(dev[2], dX)
    assert np.all(np.abs(f64(acc) - 2 * rw) <= 2 * tol_w + 2.0 ** -23 * np.abs(rw))


def test_norm_gradient_by_differences(mf):
    """dX and dw against central differences of the kernel's own fp32 forward."""
    t = torch()
    T, h, e = 3, 128, 2.0 ** -7
    g = gen(9)
    X, w, dY = (draw(g, *s).cuda() for s in ((T, h), (h,), (T, h)))
    dX, dw = nan_out((T, h), X), nan_out((h,), X)
    mf.memfine_norm_bwd(EPS, X, w, dY, dX, dw)

    def f(x, ww):
        Y = nan_out((T, h), X)
        mf.memfine_norm_fwd(EPS, x.contiguous(), ww.contiguous(), Y=Y)
        return (Y.double() * dY.double()).sum().item()
    for i in range(4):
        d, c = draw(gen(50 + i), T, h).cuda(), draw(gen(70 + i), h).cuda()
        want = (f(X + e * d, w) - f(X - e * d, w)) / (2 * e)
        # third-order term e^2 and the forward's 2e-6 of the products' magnitude over 2 e
        tol = 400 * e * e + 2e-6 * T * h / e
        assert abs((dX.double() * d).sum().item() - want) < tol
        want = (f(X, w + e * c) - f(X, w - e * c)) / (2 * e)
        assert abs((dw.double() * c).sum().item() - want) < tol


def test_norm_of_no_rows(mf):
    t = torch()
    X = t.zeros((0, 64), dtype=t.bfloat16, device="cuda")
    w = t.ones(64, dtype=t.bfloat16, device="cuda")
    mf.memfine_norm_fwd(EPS, X, w, Y=X)
    dw = t.full((64,), 3.0, device="cuda")
    mf.memfine_norm_bwd(EPS, X, w, X, X, dw, accumulate_dw=True)
    assert t.all(dw == 3)
    mf.memfine_norm_bwd(EPS, X, w, X, X, dw)
    assert t.all(dw == 0)


# ----------------------------------------------------------------- routing
def clear_logits(T, E, k, score, bias, groups, top, seed):
    """Logits whose selection and order keep a margin of 1e-5 of the values."""
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((T, E)) * rng.uniform(0.5, 2, (T, 1))).astype(np.float32)
    for _ in range(200):
        p, _ = oa.scores(z, score)
        v = p + (0 if bias is None else bias.astype(np.float64))
        bad = np.zeros(T, bool)
        for t in range(T):
            left = v[t]
            if groups > 1:
                per = v[t].reshape(groups, -1)
                g = (-np.sort(-per, axis=1)[:, :2]).sum(axis=1)
                s = -np.sort(-g)
                bad[t] |= top < groups and s[top - 1] - s[top] < 1e-5 * np.abs(s).max()
                left = per[np.argsort(-g)[:top]].ravel()
            s = -np.sort(-left)[:k + 1]
            bad[t] |= bool(np.any(s[:-1] - s[1:] < 1e-5 * np.abs(s).max()))
        if not bad.any():
            return z
        z[bad] = rng.standard_normal((bad.sum(), E)).astype(np.float32) * 1.5
    raise AssertionError("no clear logits")


ROUTES = [  # E, k, groups, top_groups
    (1, 1, 1, 1), (3, 2, 1, 1), (8, 3, 2, 1), (16, 16, 1, 1), (37, 5, 1, 1), (60, 6, 6, 3),
    (64, 8, 8, 4), (96, 4, 3, 2), (130, 7, 10, 4), (160, 6, 8, 3), (256, 8, 8, 4),
    (256, 16, 16, 5), (255, 8, 5, 2), (64, 2, 16, 16), (16, 4, 16, 6)]


@pytest.mark.parametrize("E,k,groups,top", ROUTES)
@pytest.mark.parametrize("score,renorm,with_bias", [("softmax", True, False), ("sigmoid", True, True),
                                                    ("softmax", False, True), ("sigmoid", False, False)])
def test_route(mf, E, k, groups, top, score, renorm, with_bias):
    t = torch()
    T = 37
    rng = np.random.default_rng(E * 131 + k)
    bias = (rng.standard_normal(E) * 0.1).astype(np.float32) if with_bias else None
    z = clear_logits(T, E, k, score, bias, groups, top, E + 1000 * k)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    gating = mf.make_gating(E, k, score, groups, top, renorm, scale=1.5)
    zd = t.from_numpy(z).cuda()
    idx = t.full((T, k), -7, dtype=t.int32, device="cuda")
    gates = t.full((T, k), float("nan"), device="cuda")
    dz = t.full((T, E), float("nan"), device="cuda")
    mf.memfine_route_fwd(gating, zd, idx, gates,
                         bias=None if bias is None else t.from_numpy(bias).cuda())
    mf.memfine_route_bwd(gating, zd, idx, t.from_numpy(dg).cuda(), dz)
    ri, rg = oa.route_fwd(z, k, score, bias, groups, top, renorm, 1.5)
    assert np.array_equal(idx.cpu().numpy(), ri)
    assert np.all(np.abs(f64(gates) - rg) <= 4e-6 * rg + 1e-37)
    rz = oa.route_bwd(z, ri, dg, score, renorm, 1.5)
    p, q = oa.scores(z, score)
    g = np.take_along_axis(p, ri, axis=1) * (1 if not renorm else 1 / np.maximum(
        np.take_along_axis(p, ri, axis=1).sum(axis=1, keepdims=True), 1e-300))
    spread = 1.5 * ((np.abs(dg) * g).sum(axis=1, keepdims=True) + np.abs(dg).max(axis=1, keepdims=True))
    mag = np.zeros((T, E))
    np.put_along_axis(mag, ri, g * spread, axis=1)
    if score == "softmax" and not renorm:
        mag = p * spread
    assert np.all(np.abs(f64(dz) - rz) <= 1e-5 * mag + 1e-37)


def test_route_exact_ties_take_the_lower_id(mf):
    t = torch()
    for E, groups, top, k in ((64, 1, 1, 8), (64, 8, 3, 8), (60, 6, 2, 7), (256, 8, 4, 8)):
        rng = np.random.default_rng(E + groups)
        z = rng.integers(0, 3, (50, E)).astype(np.float32)
        for score in ("softmax", "sigmoid"):
            idx = t.zeros((50, k), dtype=t.int32, device="cuda")
            gates = t.zeros((50, k), device="cuda")
            mf.memfine_route_fwd(mf.make_gating(E, k, score, groups, top), t.from_numpy(z).cuda(),
                                 idx, gates)
            # ranked on the logits, of which both scores are increasing functions; a group's
            # two best are summed over the score's own values
            p, _ = oa.scores(z, score)
            ref = oa.select(np.round(p, 12), k, groups, top)
            assert np.array_equal(idx.cpu().numpy(), ref), (E, groups, score)


def test_route_masks(mf):
    """-inf, the lowest float and NaN mask an expert, +inf counts as the largest
    float; a token without experts gets zero gates and no gradient."""
    t = torch()
    E, k = 64, 4
    rng = np.random.default_rng(5)
    z = clear_logits(40, E, k, "sigmoid", None, 1, 1, 6)
    z[0] = -np.inf
    z[1] = np.nan
    z[2] = -oa.FLT_MAX
    z[3, 3:] = -np.inf                         # fewer than k left
    z[4, ::2] = np.nan
    z[5, 5] = np.inf
    z[6] = -200.0                              # every sigmoid underflows
    z[6, 9] = -150.0
    z[7, 1:] = -oa.FLT_MAX
    for score, renorm, groups, top in itertools.product(("softmax", "sigmoid"), (True, False),
                                                        (1, 4), (1,)):
        gating = mf.make_gating(E, k, score, groups, max(top, groups // 2), renorm)
        zd = t.from_numpy(z).cuda()
        idx = t.full((40, k), -7, dtype=t.int32, device="cuda")
        gates = t.full((40, k), float("nan"), device="cuda")
        dz = t.full((40, E), float("nan"), device="cuda")
        mf.memfine_route_fwd(gating, zd, idx, gates)
        mf.memfine_route_bwd(gating, zd, idx, t.ones((40, k), device="cuda"), dz)
        i, g, d = idx.cpu().numpy(), f64(gates), f64(dz)
        assert np.all(np.isfinite(g)) and np.all(np.isfinite(d)) and np.all((i >= 0) & (i < E))
        assert np.all(g[:3] == 0) and np.all(d[:3] == 0)
        assert all(len(set(r)) == k for r in i.tolist())
        if groups == 1:
            assert set(i[3, :3]) == {0, 1, 2} and i[3, 3] == 3 and g[3, 3] == 0
        assert np.all(i[4] % 2 == 1)
        assert groups > 1 or 5 in i[5]
        assert i[7, 0] == 0 and np.all(g[7, 1:] == 0)
        assert np.all(d[oa.masked(z)] == 0)
        if groups == 1:
            # the order of underflowing scores is that of the fp32 scores: compare the others
            ri, rg = oa.route_fwd(z, k, score, None, 1, 1, renorm, 1.0)
            rows = [r for r in range(40) if r != 6]
            assert np.array_equal(i[rows], ri[rows])
            assert np.all(np.abs(g[rows] - rg[rows]) <= 4e-6 * rg[rows] + 1e-37)


def test_route_dropped_and_repeated_slots_backward(mf):
    t = torch()
    T, E, k = 33, 40, 5
    rng = np.random.default_rng(8)
    z = rng.standard_normal((T, E)).astype(np.float32)
    idx = rng.integers(0, 6, (T, k)).astype(np.int32)     # many repeats
    idx[::3, 1] = -1
    idx[::4, 2] = E
    dg = rng.standard_normal((T, k)).astype(np.float32)
    for score, renorm in itertools.product(("softmax", "sigmoid"), (True, False)):
        dz = t.full((T, E), float("nan"), device="cuda")
        mf.memfine_route_bwd(mf.make_gating(E, k, score, renorm=renorm), t.from_numpy(z).cuda(),
                             t.from_numpy(idx).cuda(), t.from_numpy(dg).cuda(), dz)
        ref = oa.route_bwd(z, idx, dg, score, renorm)
        assert np.max(np.abs(f64(dz) - ref)) <= 1e-5 * np.abs(dg).max() * 2


@pytest.mark.parametrize("T", (1, 15, 16, 17, 4097))
def test_route_any_number_of_tokens(mf, T):
    """Rows past the last token are not touched, and each token is its own."""
    t = torch()
    E, k = 160, 6
    z = t.randn(T, E, generator=gen(T)).cuda()
    gating = mf.make_gating(E, k, "sigmoid", 8, 3, True, 2.5)
    big_i = t.full((T + 16, k), -7, dtype=t.int32, device="cuda")
    big_g = t.full((T + 16, k), -7.0, device="cuda")
    big_d = t.full((T + 16, E), -7.0, device="cuda")
    mf.memfine_route_fwd(gating, z, big_i[:T], big_g[:T])
    mf.memfine_route_bwd(gating, z, big_i[:T], big_g[:T], big_d[:T])
    assert t.all(big_i[T:] == -7) and t.all(big_g[T:] == -7) and t.all(big_d[T:] == -7)
    i1, g1 = t.zeros((1, k), dtype=t.int32, device="cuda"), t.zeros((1, k), device="cuda")
    for r in {0, T // 2, T - 1}:
        mf.memfine_route_fwd(gating, z[r:r + 1], i1, g1)
        assert t.equal(i1[0], big_i[r]) and t.equal(g1[0], big_g[r])


def test_calls_run_on_the_stream_they_are_given(mf):
    """A call enqueued on a side stream sees what that stream wrote before it."""
    t = torch()
    side = t.cuda.Stream()
    T, h = 512, 1024
    src = t.randn(T, h, generator=gen(1)).to(t.bfloat16).cuda()
    w = t.ones(h, dtype=t.bfloat16, device="cuda")
    ref = nan_out((T, h), src)
    mf.memfine_norm_fwd(EPS, src, w, Y=ref)
    t.cuda.synchronize()
    X, Y = t.zeros_like(src), nan_out((T, h), src)
    t.cuda.synchronize()
    with t.cuda.stream(side):
        for _ in range(20):
            X.copy_(src)
        mf.memfine_norm_fwd(EPS, X, w, Y=Y)
    side.synchronize()
    assert t.equal(Y, ref)


# -------------------------------------------------- the router's own product
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,h,E", [(1, 64, 1), (33, 576, 37), (300, 512, 64), (257, 1024, 160),
                                   (129, 640, 250), (600, 512, 256)])
def test_router_logits_and_gradients(mf, T, h, E, dtype):
    """Against float64 products of the stored inputs, at the tolerances of the
    router's tests (2e-2 bf16, 1e-4 fp32 of the largest value)."""
    t = torch()
    g = gen(T + E)
    X, Wr = draw(g, T, h, dtype=dtype), draw(g, E, h, dtype=dtype, std=h ** -0.5)
    dl = draw(g, T, E)
    shape = mf.make_shape(T, h, 64, E, 1, mf.BF16 if dtype == "bf16" else mf.F32)
    z = t.full((T, E), float("nan"), device="cuda")
    mf.memfine_router_logits(shape, X.cuda(), Wr.cuda(), z)
    tol = 2e-2 if dtype == "bf16" else 1e-4
    ref = f64(X) @ f64(Wr).T
    assert np.max(np.abs(f64(z) - ref)) <= tol * np.max(np.abs(ref))
    base = draw(g, T, h, dtype=dtype)
    for acc in (False, True):
        dX = base.cuda() if acc else nan_out((T, h), X)
        dWr = t.full((E, h), 2.0 if acc else float("nan"), device="cuda")
        mf.memfine_router_logits_bwd(shape, X.cuda(), Wr.cuda(), dl.cuda(), dX, dWr,
                                     accumulate_dX=acc, accumulate_dWr=acc)
        rX = f64(dl) @ f64(Wr) + (f64(base) if acc else 0)
        rW = f64(dl).T @ f64(X) + (2.0 if acc else 0)
        assert np.max(np.abs(f64(dX) - rX)) <= tol * np.max(np.abs(rX))
        assert np.max(np.abs(f64(dWr) - rW)) <= tol * np.max(np.abs(rW))


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_route_agrees_with_the_router(mf, dtype):
    """Renormalised softmax top-k from the logits is the router's own routing,
    and its gradient the router's."""
    t = torch()
    T, h, E, k = 200, 512, 64, 6
    g = gen(4)
    X, Wr = draw(g, T, h, dtype=dtype).cuda(), draw(g, E, h, dtype=dtype, std=h ** -0.5).cuda()
    shape = mf.make_shape(T, h, 64, E, k, mf.BF16 if dtype == "bf16" else mf.F32)
    idx, idx2 = (t.zeros((T, k), dtype=t.int32, device="cuda") for _ in range(2))
    gates, gates2 = (t.zeros((T, k), device="cuda") for _ in range(2))
    z, z2 = (t.zeros((T, E), device="cuda") for _ in range(2))
    mf.memfine_router_fwd(shape, X, Wr, idx, gates, z)
    mf.memfine_router_logits(shape, X, Wr, z2)
    assert t.equal(z, z2)
    gating = mf.make_gating(E, k)
    mf.memfine_route_fwd(gating, z, idx2, gates2)
    ref = orr.topk(z.cpu().numpy(), k)
    assert np.array_equal(idx.cpu().numpy(), ref)
    same = (idx == idx2).all(1)
    assert same.float().mean() > 0.98          # (equal scores of different logits may swap)
    assert t.allclose(gates[same], gates2[same], rtol=1e-5, atol=1e-7)
    dg = draw(g, T, k).cuda()
    dz = t.zeros((T, E), device="cuda")
    mf.memfine_route_bwd(gating, z, idx, dg, dz)
    rz = orr.router_bwd(f64(X), f64(Wr), idx.cpu().numpy(), f64(z), f64(dg))["dlogits"]
    assert np.max(np.abs(f64(dz) - rz)) <= 1e-5 * np.max(np.abs(rz))
