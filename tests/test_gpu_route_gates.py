"""Gates and gradients of experts far below the best one, which a bias selects.

The logits are multiples of 2^-8 below 2^7 in size, so their differences are
exact floats.  Relative errors, in units of u = 2^-24, from the arithmetic: an
exponential 4 (its unit of 2, the remainder's factor, the last fma); a softmax's
sum of E <= 32 terms 8 (4 from the terms, of which those that count are near
the largest; 1 + 4 additions, of positive numbers whose largest is 1, lose at most
half a unit of 2^-23 each: 3) and its reciprocal 1; a sigmoid's reciprocal of 1 + e
3; a product 1.  Gates: 16.  Renormalised: score 8, sum 12, quotient and scale 3: 24.
Gradients of unrenormalised softmax gates c p_e: c 16 + 6 (products, additions),
p_e 16, product 1: 40; of a renormalised or sigmoid gate: 40 of the sum of the
magnitudes that it is formed from.
"""
import numpy as np
import pytest

from gpu_harness import torch
from oracle import around as oa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mf():
    t = torch()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_21431_amd as m
    m.lib()
    return m


def f64(x):
    return x.detach().cpu().double().numpy()


def case(score, E, k, seed):
    """Logits from 0 down to -87; the bias takes the first k experts."""
    rng = np.random.default_rng(seed)
    T = 301
    z = -np.floor(rng.uniform(0, 87, (T, E)) * 256) / 256
    z[:, -1] = 0.0
    bias = np.zeros(E)
    bias[:k] = 8 - np.arange(k)
    return T, z, bias


@pytest.mark.parametrize("renorm", (False, True))
@pytest.mark.parametrize("E,k", ((8, 1), (16, 4), (32, 8)))
@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
def test_small_gates(mf, score, E, k, renorm):
    t = torch()
    T, z, bias = case(score, E, k, E + k)
    gating = mf.make_gating(E, k, score, renorm=renorm)
    zd, bd = (t.from_numpy(a.astype(np.float32)).cuda() for a in (z, bias))
    idx, gates = t.zeros((T, k), dtype=t.int32, device="cuda"), t.zeros((T, k), device="cuda")
    mf.memfine_route_fwd(gating, zd, idx, gates, bias=bd)
    want = np.tile(np.arange(k, dtype=np.int32), (T, 1))
    assert np.array_equal(idx.cpu().numpy(), want)
    ref = oa.gates_of(oa.scores(z, score)[0], want, renorm, 1.0)
    assert np.all(np.abs(f64(gates) - ref) <= (24 if renorm else 16) * U * ref)
    # gradients, of positive dgates: nothing cancels in the unrenormalised ones
    dg = np.abs(np.random.default_rng(1).standard_normal((T, k))).astype(np.float32)
    d = t.full((T, E), 5.0, device="cuda")
    mf.memfine_route_bwd(gating, zd, idx, t.from_numpy(dg).cuda(), d)
    rd = oa.route_bwd(z, want, dg.astype(np.float64), score, renorm, 1.0)
    mag = np.zeros((T, E))
    p = oa.scores(z, score)[0]
    if renorm:
        comp = 1.0 if score == "softmax" else 1.0 / (1.0 + np.exp(z[:, :k]))
        mag[:, :k] = ref * comp * (dg + (ref * dg).sum(axis=1, keepdims=True))
    elif score == "softmax":
        mag = p * (p[:, :k] * dg).sum(axis=1, keepdims=True)
        mag[:, :k] += p[:, :k] * dg
    else:
        mag = np.abs(rd)
    small = mag < 2.0 ** -120      # near or below the smallest float
    assert np.all((np.abs(f64(d) - rd) <= 40 * U * mag)[~small])
    assert np.all(np.abs(f64(d) - rd)[small] <= 2.0 ** -119)
