"""More rows than one launch holds (2^32 work-items): the calls around the
layer give every row what it gets in a small call."""
import numpy as np
import pytest

from gpu_harness import log, torch
from test_gpu_mxw import activations, mf, packed, rows  # noqa: F401

pytestmark = pytest.mark.gpu


def room(gib):
    t = torch()
    t.cuda.empty_cache()
    if t.cuda.mem_get_info()[0] < gib * 2**30:
        pytest.skip(f"needs {gib} GiB of device memory")


def repeated(x, T):
    """Rows x, repeated up to T rows."""
    t, n = torch(), x.shape[0]
    big = t.empty((T, *x.shape[1:]), dtype=x.dtype, device="cuda")
    whole = T // n * n
    big[:whole].view(T // n, *x.shape).copy_(x)
    big[whole:] = x[:T - whole]
    return big


def repeats(big, x):
    """Whether big is x's rows, repeated (compared a part at a time)."""
    t, n = torch(), x.shape[0]
    whole = big.shape[0] // n * n
    parts = big[:whole].view(-1, *x.shape)
    step = max(1, 2**31 // x.numel())
    return all(bool((parts[i:i + step] == x).all()) for i in range(0, len(parts), step)) \
        and t.equal(big[whole:], x[:big.shape[0] - whole])


def test_norm(mf):
    room(40)
    t = torch()
    T, h, n = 2**26 + 37, 64, 4099
    X, R = (t.randn(n, h, device="cuda").to(t.bfloat16) for _ in range(2))
    w = t.randn(h, device="cuda").to(t.bfloat16)
    small = [t.empty_like(X), t.empty_like(X), t.zeros(n, h, dtype=t.uint8, device="cuda"),
             t.zeros(n, h // 32, dtype=t.uint8, device="cuda")]
    mf.memfine_norm_fwd(1e-6, X, w, R=R, S=small[0], Y=small[1], Q=small[2], QS=small[3])
    X, R = repeated(X, T), repeated(R, T)
    out = [t.zeros((T, *x.shape[1:]), dtype=x.dtype, device="cuda") for x in small]
    log("norm", T)
    mf.memfine_norm_fwd(1e-6, X, w, R=R, S=out[0], Y=out[1], Q=out[2], QS=out[3])
    assert all(repeats(a, b) for a, b in zip(out, small))
    Y = out[1].zero_()
    mf.memfine_norm_fwd(1e-6, X, w, Y=Y)
    mf.memfine_norm_fwd(1e-6, X[:n], w, Y=small[1])
    assert repeats(Y, small[1])


def test_route(mf):
    room(16)
    t = torch()
    T, E, k, n = 2**28 + 37, 2, 1, 4099
    z = t.randn(n, E, device="cuda")
    gating = mf.make_gating(E, k, renorm=False)
    idx, gates, dz = (t.zeros(n, k, dtype=t.int32, device="cuda"), t.zeros(n, k, device="cuda"),
                      t.zeros(n, E, device="cuda"))
    mf.memfine_route_fwd(gating, z, idx, gates)
    mf.memfine_route_bwd(gating, z, idx, gates, dz)
    z = repeated(z, T)
    I, G = t.full((T, k), -1, dtype=t.int32, device="cuda"), t.zeros(T, k, device="cuda")
    log("route", T)
    mf.memfine_route_fwd(gating, z, I, G)
    assert repeats(I, idx) and repeats(G, gates)
    D = t.zeros(T, E, device="cuda")
    mf.memfine_route_bwd(gating, z, I, G, D)
    assert repeats(D, dz)


def test_mx_values(mf):
    room(112)
    t = torch()
    T, h, n = 2**21 + 5, 16384, 1021
    q = t.randint(0, 0x7f, (n, h), dtype=t.uint8, device="cuda")
    qs = t.randint(100, 140, (n, h // 32), dtype=t.uint8, device="cuda")
    small = t.zeros(n, h, dtype=t.bfloat16, device="cuda")
    mf.memfine_mx_values(q, qs, small)
    q, qs = repeated(q, T), repeated(qs, T)
    out = t.zeros(T, h, dtype=t.bfloat16, device="cuda")
    log("values", T, h)
    mf.memfine_mx_values(q, qs, out)
    assert repeats(out, small)


def test_pack(mf):
    room(160)
    t = torch()
    E, N, K, n = 2**9 + 3, 2**14, 2**14, 37
    rc = t.randint(0, 256, (n, N, K // 2), dtype=t.uint8, device="cuda")
    rs = t.randint(100, 140, (n, N, K // 32), dtype=t.uint8, device="cuda")
    c, s = mf.memfine_mxw_pack(n, N, K, rc, rs)
    rc, rs = repeated(rc, E), repeated(rs, E)
    log("pack", E, N, K)
    C, S = mf.memfine_mxw_pack(E, N, K, rc, rs)
    assert repeats(C, c) and repeats(S, s)


@pytest.mark.parametrize("mx8", (False, True))
def test_linear(mf, mx8):
    """2^30 rows, which one launch of tiles of 64 rows does not hold."""
    room(112)
    t = torch()
    rng = np.random.default_rng(5)
    T, N, K, n = 2**30 + 37, 16, 32, 65537
    W = packed(mf, 1, N, K, *rows(rng, 1, N, K)[:2])
    X, XS, _ = activations(rng, n, K, mx8)
    small = t.zeros(n, N, dtype=t.bfloat16, device="cuda")
    mf.memfine_linear_mxw(N, K, X, *W, small, XS=XS)
    X, XS = repeated(X, T), None if XS is None else repeated(XS, T)
    Y = t.zeros(T, N, dtype=t.bfloat16, device="cuda")
    log("linear", T, mx8)
    mf.memfine_linear_mxw(N, K, X, *W, Y, XS=XS)
    assert repeats(Y, small)
