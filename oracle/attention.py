"""Oracle of the attention in front of the layer, plain fp64 NumPy (test
infrastructure only): packed sequences and their gradient, one token over a
cache, rotation by position.  Definitions are those of include/memfine.h; pinned
by tests/test_oracle_attention.py (loops over pairs, finite differences, complex
numbers).

Beside each result stand the sums of magnitudes that bound its rounding errors.
"""
from __future__ import annotations

import numpy as np


def _f64(a) -> np.ndarray:
    return np.asarray(a, dtype=np.float64)


def sees(n, causal, window=0) -> np.ndarray:
    """[n, n], true where token i sees token j."""
    i, j = np.arange(n)[:, None], np.arange(n)
    m = (j <= i) if causal else np.ones((n, n), bool)
    return m & (j > i - window) if window else m


def weights(S, mask):
    """(softmax over the tokens seen, its lse); zeros and -inf where none is."""
    S = np.where(mask, S, -np.inf)
    m = S.max(axis=-1, keepdims=True, initial=-np.inf)
    e = np.where(mask, np.exp(S - np.where(np.isfinite(m), m, 0.0)), 0.0)
    t = e.sum(axis=-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(t))[..., 0]
    return np.divide(e, t, out=np.zeros_like(e), where=t > 0), lse


def one_fwd(q, k, v, scale, mask):
    """One head of one sequence: O, lse, and sum_j p |v_j|, max_j scale sum |q k|."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    p, lse = weights(scale * (q @ k.T), mask)
    big = np.where(mask, scale * (np.abs(q) @ np.abs(k).T), 0.0).max(axis=1, initial=0.0)
    return p @ v, lse, p @ np.abs(v), big


def one_bwd(q, k, v, o, lse, do, scale, mask):
    """One head of one sequence: p, ds and the arrays that their errors come from:
    |dp| and |delta| as sums of magnitudes, s."""
    q, k, v, o, do = map(_f64, (q, k, v, o, do))
    s = scale * (q @ k.T)
    lse = _f64(lse)[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(mask & np.isfinite(lse), np.exp(np.where(mask, s - lse, 0.0)), 0.0)
    dp, delta = do @ v.T, (do * o).sum(axis=1, keepdims=True)
    ds = scale * p * (dp - delta)
    mag = np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(axis=1, keepdims=True)
    return p, ds, np.abs(dp) + np.abs(delta), mag, np.where(mask, np.abs(s), 0.0)


def packed(offsets, T):
    """(first row, length) of the sequences."""
    return [(int(a), int(b) - int(a)) for a, b in zip(offsets[:-1], offsets[1:])]


def attn_fwd(Q, K, V, offsets, scale, causal, window=0):
    """O [T, heads, dim], lse [heads, T] and their bounds' sums, NaN in rows of no
    sequence."""
    Q, K, V = map(_f64, (Q, K, V))
    T, H, D = Q.shape
    g = H // K.shape[1]
    O, A = np.full((T, H, D), np.nan), np.full((T, H, D), np.nan)
    lse, big = np.full((H, T), np.nan), np.full((H, T), np.nan)
    for at, n in packed(offsets, T):
        r = slice(at, at + n)
        m = sees(n, causal, window)
        for h in range(H):
            O[r, h], lse[h, r], A[r, h], big[h, r] = one_fwd(Q[r, h], K[r, h // g], V[r, h // g],
                                                             scale, m)
    return O, lse, A, big


def attn_bwd(Q, K, V, O, lse, dO, offsets, scale, causal, window=0, rounding=0.0, unit=0.0):
    """dQ, dK, dV and the bounds of their errors, for weights and ds that are rounded by
    `rounding` of their value and fp32 arithmetic of `unit` a step."""
    Q, K, V, O, dO = map(_f64, (Q, K, V, O, dO))
    T, H, D = Q.shape
    Hk = K.shape[1]
    out = [np.zeros_like(x) for x in (Q, K, V)]
    err = [np.zeros_like(x) for x in (Q, K, V)]
    for at, n in packed(offsets, T):
        r = slice(at, at + n)
        m = sees(n, causal, window)
        for h in range(H):
            y = h // (H // Hk)
            q, k, v, do = Q[r, h], K[r, y], V[r, y], dO[r, h]
            p, ds, dp, mag, s = one_bwd(q, k, v, O[r, h], lse[h, r], do, scale, m)
            out[0][r, h] = ds @ k
            out[1][r, y] += ds.T @ q
            out[2][r, y] += p.T @ do
            # relative error of a weight: its score's sum, the lse's product, the power
            pe = unit * (4 * (s + np.abs(np.where(np.isfinite(lse[h, r]), lse[h, r], 0.0))[:, None])
                         + (D + 4) * scale * (np.abs(q) @ np.abs(k).T) + 8)
            de = rounding * np.abs(ds) + scale * p * (pe * dp + unit * (D + 8) * mag)
            # the products' own sums: a step a term
            ve = p * (rounding + pe + unit * (n + 8))
            de = de + np.abs(ds) * unit * (n * (H // Hk) + 8)
            err[0][r, h] = de @ np.abs(k)
            err[1][r, y] += de.T @ np.abs(q)
            err[2][r, y] += (ve + unit * n * (H // Hk) * p).T @ np.abs(do)
    return out, err


def decode(q, k, v, scale, window=0):
    """The last token's O [heads, dim] over k, v [n, kv_heads, dim], lse, bounds' sums."""
    q, k, v = map(_f64, (q, k, v))
    H, D = q.shape
    n, Hk = k.shape[:2]
    O, A = np.zeros((H, D)), np.zeros((H, D))
    lse, big = np.full(H, -np.inf), np.zeros(H)
    lo = max(0, n - window) if window else 0
    if n > 0:
        for h in range(H):
            y = h // (H // Hk)
            o, l, a, b = one_fwd(q[h][None], k[lo:, y], v[lo:, y], scale, np.ones((1, n - lo), bool))
            O[h], lse[h], A[h], big[h] = o[0], l[0], a[0], b[0]
    return O, lse, A, big


def rope(X, cos, sin, interleaved=False, inverse=False):
    """Rows X [T, heads, dim] turned by the rows' cos and sin [T, dim / 2], and the
    sums of magnitudes."""
    X, c, s = _f64(X), _f64(cos)[:, None], _f64(sin)[:, None]
    s = -s if inverse else s
    if interleaved:
        a, b = X[..., 0::2], X[..., 1::2]
    else:
        a, b = np.split(X, 2, axis=-1)
    ya, yb = a * c - b * s, b * c + a * s
    ma, mb = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    out, mag = np.empty_like(X), np.empty_like(X)
    half = X.shape[-1] // 2
    for y, (u, w) in ((out, (ya, yb)), (mag, (ma, mb))):
        if interleaved:
            y[..., 0::2], y[..., 1::2] = u, w
        else:
            y[..., :half], y[..., half:] = u, w
    return out, mag
