"""MX4 products with the ends of the scale bytes, in every kernel that
multiplies: 0 stands for 2^-127, 255 marks a block whose values are all NaN,
zero codes among them.

Tolerances are those of test_gpu_mxw_kernels.py; the small scales meet
activations that are large enough for the products to be ordinary floats.
"""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from test_gpu_mxw import activations, check, dev, experts_case, f64, mf, packed, rows  # noqa: F401
from test_gpu_mxw_kernels import bound

pytestmark = pytest.mark.gpu

# one row, few rows (short and split reductions), tiles of 32, 64 and 128 rows
LINEAR = [(1, 64, 672), (1, 4096, 160), (5, 64, 672), (5, 64, 4640), (40, 96, 4640), (600, 1040, 160),
          (1100, 4112, 160), (2049, 4112, 96), (4224, 16384, 96)]


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,N,K", LINEAR)
def test_linear_smallest_scale(mf, T, N, K, mx8):
    """Rows 3 mod 16 of W have scale byte 0 in every block, 5 mod 16 have 1."""
    t = torch()
    rng = np.random.default_rng(T + N + K)
    c, s, _ = rows(rng, 1, N, K)
    s[0, 3::16], s[0, 5::16] = 0, 1
    W = np.where(c_bits(c) >= 8, -1.0, 1.0) * oa.E2M1[c_bits(c) & 7]
    W = W[0] * np.repeat(2.0 ** (s[0] - 127.0), 32, axis=1)
    codes, scales = packed(mf, 1, N, K, c, s)
    log(f"smallest scale T={T} N={N} K={K} mx8={mx8}")
    X, XS, x = activations(rng, T, K, mx8, 2.0 ** 60)
    Y = t.full((T, N), float("nan"), device="cuda")
    mf.memfine_linear_mxw(N, K, X, codes, scales, Y, XS=XS)
    pick = np.unique(np.concatenate([rng.integers(0, T, 40), np.arange(min(T, 40))]))
    ref, tol = bound(x[pick], W, mx8)
    got = f64(Y[t.from_numpy(pick).cuda()])
    assert np.all(np.abs(got - ref) <= tol)
    assert np.all(got[:, 3::16].any(axis=1))


def c_bits(c):
    return np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,N,K", LINEAR)
def test_linear_block_of_nans(mf, T, N, K, mx8):
    """Scale byte 255, once over zero codes: NaN in those columns, the others
    as without."""
    t = torch()
    rng = np.random.default_rng(T * N + K)
    c, s, _ = rows(rng, 1, N, K)
    clean, Y = (t.full((T, N), 7.0, device="cuda") for _ in range(2))
    X, XS, x = activations(rng, T, K, mx8)
    bad = np.array([2, 17, N - 1])
    c[0, 17, :16] = 0                       # codes of the first block
    c[0, N - 1, -16:] = 0x88                # -0 in the last
    log(f"block of NaNs T={T} N={N} K={K} mx8={mx8}")
    codes, scales = packed(mf, 1, N, K, c, s)
    mf.memfine_linear_mxw(N, K, X, codes, scales, clean, XS=XS)
    s[0, 2, K // 64] = s[0, 17, 0] = s[0, N - 1, -1] = 255
    codes, scales = packed(mf, 1, N, K, c, s)
    mf.memfine_linear_mxw(N, K, X, codes, scales, Y, XS=XS)
    keep = np.setdiff1d(np.arange(N), bad)
    assert t.all(t.isnan(Y[:, t.from_numpy(bad).cuda()]))
    keep = t.from_numpy(keep).cuda()
    assert t.all(t.isfinite(clean)) and t.equal(Y[:, keep], clean[:, keep])


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,h,F,E,k", [(1, 256, 256, 3, 2), (2, 256, 256, 3, 2), (700, 256, 256, 3, 2),
                                       (4100, 64, 4096, 3, 2), (4100, 1088, 1024, 4, 3)])
def test_experts_block_of_nans(mf, T, h, F, E, k, mx8):
    """One block of 255 in expert 0's W1 makes the tokens that have it NaN; in
    its W2, one column of theirs."""
    t = torch()
    rng = np.random.default_rng(T + F)
    (c1, s1, _), (c2, s2, _), X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, mx8)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    idx[0, 0], idx[0, 1:] = 0, np.arange(1, k)
    has = t.from_numpy((idx == 0).any(axis=1)).cuda()
    log(f"experts' block of NaNs T={T} h={h} F={F} mx8={mx8}")

    def run(s1, s2):
        p1, p2 = packed(mf, E, 2 * F, h, c1, s1), packed(mf, E, h, F, c2, s2)
        Y = t.zeros((T, h), dtype=t.bfloat16, device="cuda")
        mf.memfine_moe_fwd_mxw(mf.make_shape(T, h, F, E, k, mf.BF16), 1, X, dev(idx), dev(g), *p1,
                               *p2, Y, XS=XS)
        return Y
    c1[0, F + 9, 16:32] = 0
    clean = run(s1, s2)
    s1[0, F + 9, 1] = 255
    Y = run(s1, s2)
    assert t.all(t.isfinite(clean)) and t.all(t.isnan(Y[has])) and t.equal(Y[~has], clean[~has])
    s1[0, F + 9, 1] = 120
    clean = run(s1, s2)
    s2[0, 21, F // 32 - 1] = 255
    Y = run(s1, s2)
    bad = t.zeros((T, h), dtype=t.bool, device="cuda")
    bad[has, 21] = True
    assert t.all(t.isnan(Y[bad])) and t.equal(Y[~bad], clean[~bad])
