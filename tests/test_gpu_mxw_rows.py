"""The rows between the experts' second product and the sum over a token's slots:
they add nothing visible to Y's own rounding, however many they are and however
the call is cut into chunks.

Y in bf16 alone is off by 2^-7 / sqrt(12) of the power of two below each value, 1.5e-3
to 1.7e-3 of the 2-norm; rows kept to 2^-12 add an eighth of that in quadrature (the
k slots of a token weigh at most as much as Y), 1 %, and the products' cut on MX8
2e-4.  1.9e-3 in all, where rows of bf16 add as much as Y's rounding, 2.3e-3."""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from test_gpu_mxw import dev, experts_case, f64, mf, packed, rows, run_experts  # noqa: F401

pytestmark = pytest.mark.gpu


def off(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("T,h,F,E,k", [(1200, 576, 1024, 4, 4), (2100, 1088, 1024, 3, 2),
                                       (700, 512, 1024, 40, 8), (5000, 192, 1024, 2, 1)])
def test_rows_add_nothing_visible(mf, T, h, F, E, k):
    rng = np.random.default_rng(T + h)
    m1, m2, X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, True)
    g = g + np.float32(0.5)
    idx[3], idx[8, 0] = -1, E
    pick = np.unique(np.concatenate([rng.integers(0, T, 200), np.arange(20), np.arange(T - 40, T)]))
    on = (idx >= 0) & (idx < E)
    ref = oa.moe_fwd_mx(x[pick], np.where(on, idx, 0)[pick], np.where(on, g, 0)[pick], m1[2], m2[2], True)
    for chunks in (1, 2, 3):
        log("rows", T, h, F, E, k, chunks)
        Y = run_experts(mf, T, h, F, E, k, (m1, m2), X, XS, idx, g, chunks=chunks)
        assert torch().all(Y[3] == 0)
        assert off(f64(Y[torch().from_numpy(pick).cuda()]), ref) <= 1.9e-3


def test_rows_of_many_sizes(mf):
    """Columns of very different sizes, each to the same precision unless they lie
    more than 2^30 below another of their 64, which leaves 2^-41 of that; an
    overflowing one changes no other."""
    t = torch()
    rng = np.random.default_rng(13)
    T, h, F, E, k = 2500, 256, 1024, 3, 2
    (c1, s1, W1), (c2, s2, W2), X, XS, x, idx, g = experts_case(rng, T, h, F, E, k, True)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    move = np.zeros(h, dtype=np.int64)          # powers of two by column
    move[64:128] = -100                         # a whole block far down
    move[128:192] = 100                         # and far up
    move[5], move[130], move[135], move[200:210] = -20, -20, 75, -12
    s2 = (s2.astype(np.int64) + move[None, :, None]).astype(np.uint8)
    W2 = W2 * 2.0 ** move[None, :, None]
    ref = oa.moe_fwd_mx(x, idx, g, W1, W2, True)
    Y = f64(run_experts(mf, T, h, F, E, k, ((c1, s1, W1), (c2, s2, W2)), X, XS, idx, g))
    assert np.all(np.isfinite(Y))
    for c in (0, 5, 64, 127, 128, 135, 191, 200, 209, 255):
        assert off(Y[:, c], ref[:, c]) <= 1.9e-3, c
    # (k slots, and a slot's row may be larger than their sum)
    assert np.max(np.abs(Y[:, 130] - ref[:, 130])) <= k * 2.0 ** -40 * np.max(np.abs(ref[:, 128:192]))
    # one column of expert 0 overflows fp32: its tokens have no number there and the others
    # of the row, in the same 64 columns, are what they were
    s2[0, 7] = 254
    has = (idx == 0).any(axis=1)
    Z = f64(run_experts(mf, T, h, F, E, k, ((c1, s1, W1), (c2, s2, W2)), X, XS, idx, g))
    assert not np.any(np.isfinite(Z[has, 7])) and np.array_equal(Z[~has, 7], Y[~has, 7])
    keep = np.arange(h) != 7
    assert off(Z[:, keep][:, :63], Y[:, keep][:, :63]) <= 1e-3
    assert np.array_equal(Z[:, 64:], Y[:, 64:])
