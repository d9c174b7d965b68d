"""The attention oracle against loops over pairs, finite differences and complex
numbers."""
import math

import numpy as np
import pytest

from oracle import attention as at


def case(lens, H, Hk, D, seed=0):
    rng = np.random.default_rng(seed)
    T = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)])
    return (rng.standard_normal((T, H, D)), rng.standard_normal((T, Hk, D)),
            rng.standard_normal((T, Hk, D)), off)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 3)])
def test_forward_against_loops(causal, window):
    Q, K, V, off = case([4, 0, 1, 6], 4, 2, 5)
    O, lse, A, big = at.attn_fwd(Q, K, V, off, 0.3, causal, window)
    for b in range(4):
        for i in range(off[b], off[b + 1]):
            for h in range(4):
                js = [j for j in range(off[b], off[b + 1])
                      if (not causal or j <= i) and (not window or j > i - window)]
                s = [0.3 * float(Q[i, h] @ K[j, h // 2]) for j in js]
                t = sum(math.exp(x) for x in s)
                assert lse[h, i] == pytest.approx(math.log(t), abs=1e-12)
                o = sum(math.exp(x) / t * V[j, h // 2] for x, j in zip(s, js))
                assert np.allclose(O[i, h], o, atol=1e-12)
                assert np.all(A[i, h] >= np.abs(o) - 1e-12)
                assert big[h, i] >= max(abs(x) for x in s) - 1e-12


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 2)])
def test_gradient_against_differences(causal, window):
    Q, K, V, off = case([3, 1, 5], 4, 2, 3, 1)
    dO = np.random.default_rng(2).standard_normal(Q.shape)
    O, lse, _, _ = at.attn_fwd(Q, K, V, off, 0.5, causal, window)
    (dQ, dK, dV), err = at.attn_bwd(Q, K, V, O, lse, dO, off, 0.5, causal, window)
    assert all(np.all(e >= 0) for e in err)

    def loss():
        return float((at.attn_fwd(Q, K, V, off, 0.5, causal, window)[0] * dO).sum())
    rng = np.random.default_rng(3)
    for x, d in ((Q, dQ), (K, dK), (V, dV)):
        for i in rng.choice(x.size, 12, replace=False):
            i = np.unravel_index(i, x.shape)
            keep, e = x[i], 1e-5
            x[i] = keep + e
            up = loss()
            x[i] = keep - e
            down = loss()
            x[i] = keep
            assert d[i] == pytest.approx((up - down) / (2 * e), abs=1e-7)


def test_rows_that_see_nothing():
    p, lse = at.weights(np.ones((2, 3)), np.array([[True, False, True], [False] * 3]))
    assert np.allclose(p, [[0.5, 0, 0.5], [0, 0, 0]]) and lse[1] == -np.inf


def test_decode_is_the_last_row():
    Q, K, V, off = case([9], 6, 2, 4, 5)
    for w in (0, 1, 4, 9, 20):
        O, lse, _, _ = at.attn_fwd(Q, K, V, off, 0.7, True, w)
        o, l, _, _ = at.decode(Q[-1], K, V, 0.7, w)
        assert np.allclose(o, O[-1]) and np.allclose(l, lse[:, -1])
    o, l, _, _ = at.decode(Q[-1], K[:0], V[:0], 0.7)
    assert np.all(o == 0) and np.all(l == -np.inf)


@pytest.mark.parametrize("interleaved", (False, True))
def test_rotation_as_complex_numbers(interleaved):
    rng = np.random.default_rng(7)
    X, a = rng.standard_normal((5, 3, 8)), rng.standard_normal((5, 4))
    y, mag = at.rope(X, np.cos(a), np.sin(a), interleaved)
    pair = (lambda x: x[..., 0::2] + 1j * x[..., 1::2]) if interleaved else \
        (lambda x: x[..., :4] + 1j * x[..., 4:])
    assert np.allclose(pair(y), pair(X) * np.exp(1j * a)[:, None])
    back, _ = at.rope(y, np.cos(a), np.sin(a), interleaved, inverse=True)
    assert np.allclose(back, X) and np.all(mag >= np.abs(y) - 1e-12)
