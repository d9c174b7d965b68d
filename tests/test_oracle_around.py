"""Pins of oracle/around.py against things other than itself: central
differences for the gradients, brute force for the selection, hand-worked MX
blocks, and torch's own float8 type for the rounding."""
import itertools

import numpy as np
import pytest
import torch

from oracle import around as oa


def difference(f, x, d, eps=1e-6):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


def test_norm_gradient_by_differences():
    rng = np.random.default_rng(0)
    X, w, dY, dS = (rng.standard_normal(s) for s in ((3, 8), (8,), (3, 8), (3, 8)))
    dX, dw = oa.norm_bwd(X, w, dY, dS, 1e-3)
    for _ in range(10):
        d = rng.standard_normal(X.shape)
        want = difference(lambda x: (oa.norm_fwd(x, w, 1e-3) * dY + x * dS).sum(), X, d)
        assert abs((dX * d).sum() - want) < 1e-7
        d = rng.standard_normal(w.shape)
        want = difference(lambda v: (oa.norm_fwd(X, v, 1e-3) * dY).sum(), w, d)
        assert abs((dw * d).sum() - want) < 1e-7


def test_norm_of_a_constant_row():
    assert np.allclose(oa.norm_fwd(np.full((1, 4), 3.0), np.arange(4.0), 0.0), [[0, 1, 2, 3]])


@pytest.mark.parametrize("score,renorm", itertools.product(("softmax", "sigmoid"), (True, False)))
def test_route_gradient_by_differences(score, renorm):
    rng = np.random.default_rng(1)
    z, dg = rng.standard_normal((4, 9)), rng.standard_normal((4, 3))
    idx, _ = oa.route_fwd(z, 3, score)
    dz = oa.route_bwd(z, idx, dg, score, renorm, 1.7)
    f = lambda z: (oa.gates_of(oa.scores(z, score)[0], idx, renorm, 1.7) * dg).sum()  # noqa: E731
    for _ in range(10):
        d = rng.standard_normal(z.shape)
        assert abs((dz * d).sum() - difference(f, z, d)) < 1e-7


def test_selection_by_brute_force():
    rng = np.random.default_rng(2)
    v = rng.integers(0, 4, (30, 12)).astype(float)   # many ties
    for groups, top in ((1, 1), (3, 2), (6, 2), (12, 5)):
        k = 3
        idx = oa.select(v, k, groups, top)
        size = 12 // groups
        for t in range(len(v)):
            g = [sum(sorted(v[t, i * size:(i + 1) * size])[-2:]) for i in range(groups)]
            # the best set of groups, and of experts: lexicographically largest (values, -ids)
            best = max(itertools.combinations(range(groups), top),
                       key=lambda c: (sorted((g[i] for i in c), reverse=True), [-i for i in c]))
            left = [e for e in range(12) if e // size in best]
            want = max(itertools.permutations(left, k),
                       key=lambda c: [(v[t, e], -e) for e in c])
            assert tuple(idx[t]) == want


def test_masked_rows():
    z = np.array([[-np.inf, np.nan, -oa.FLT_MAX, -np.inf], [1.0, -np.inf, np.inf, 0.0]])
    for score in ("softmax", "sigmoid"):
        idx, g = oa.route_fwd(z, 3, score)
        assert idx[0].tolist() == [0, 1, 2] and g[0].tolist() == [0, 0, 0]
        assert idx[1].tolist() == [2, 0, 3] and np.isclose(g[1].sum(), 1)
        assert np.all(np.isfinite(oa.route_bwd(z, idx, np.ones((2, 3)), score)))


def test_e4m3_rounding_is_torchs():
    x = np.random.default_rng(3).uniform(-448, 448, 4000).astype(np.float32)
    x = np.concatenate([x, x / 1000, oa.e4m3_values().astype(np.float32),
                        (oa.e4m3_values()[1:] + oa.e4m3_values()[:-1]).astype(np.float32) / 2])
    code, val = oa._round_to(x.astype(np.float64), oa.e4m3_values())
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(val, want.double().numpy())
    assert np.array_equal(code, want.view(torch.uint8).numpy() & 127)


def test_hand_worked_blocks():
    x = np.zeros((1, 32))
    x[0, :6] = [6.0, 0.25, 0.75, -2.5, 5.0, 1.75]
    code, s, val = oa.mx_round(x, "mx4")
    assert s.tolist() == [[127]]                       # 6 = 6 * 2^0
    assert val[0, :6].tolist() == [6, 0, 1, -2, 4, 2]  # ties to even codes
    assert code[0, :6].tolist() == [7, 0, 2, 8 + 4, 6, 4]
    x[0, 0] = 6.0001                                   # one step up: everything is halved first
    assert oa.mx_round(x, "mx4")[1].tolist() == [[128]]
    assert oa.mx_round(np.full((1, 32), 448.0), "mx8")[1].tolist() == [[127]]
    assert oa.mx_round(np.full((1, 32), 449.0), "mx8")[1].tolist() == [[128]]
    assert oa.mx_round(np.zeros((1, 32)), "mx8")[1].tolist() == [[0]]
    x[0, 3] = np.inf
    code, s, val = oa.mx_round(x, "mx8")
    assert s.tolist() == [[255]] and np.all(np.isnan(val))


def test_layout_by_index():
    rng = np.random.default_rng(4)
    E, N, K = 2, 32, 160
    c = rng.integers(0, 256, (E, N, K // 2)).astype(np.uint8)
    s = rng.integers(0, 255, (E, N, K // 32)).astype(np.uint8)
    codes, scales = oa.mx4_layout(c, s)
    assert codes.shape == (E, 2 * 2 * 1024) and scales.shape == (E, 2 * 1 * 256)
    for e, n, k in itertools.product(range(E), range(N), range(0, K, 2)):
        lane = n % 16 + 16 * (k % 128 // 32)
        at = ((n // 16 * 2 + k // 128) * 64 + lane) * 16 + k % 32 // 2
        assert codes[e, at] == c[e, n, k // 2]
        assert scales[e, (n // 16 * 64 + lane) * 4 + k // 128] == s[e, n, k // 32]


def test_mx_experts_reduce_to_the_layer_when_rounding_is_exact():
    rng = np.random.default_rng(5)
    X = rng.standard_normal((5, 64))
    W1 = np.zeros((2, 64, 64))
    W1[:, :32] = 1000.0 / 64        # silu(u) = u in double for large u ...
    W1[:, 32:] = 0.25
    X = np.abs(X) + 1
    W2 = rng.standard_normal((2, 64, 32))
    idx = rng.integers(0, 2, (5, 2)).astype(np.int32)
    g = rng.random((5, 2))
    # ... so every column of a is the same number: its MX8 value is within a sixteenth
    a = oa.moe_fwd_mx(X, idx, g, W1, W2, True)
    b = oa.moe_fwd_mx(X, idx, g, W1, W2, False)
    assert np.max(np.abs(a / b - 1)) <= 1 / 16 and np.max(np.abs(a / b - 1)) > 0
