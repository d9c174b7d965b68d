"""Oracle of what stands around the layer, plain fp64 NumPy (test
infrastructure only): the residual RMS norm and its gradient, routing from
logits and its gradient, the MX block formats, and the layer's forward with
MX4 weights.  Definitions are those of include/memfine.h; pinned by
tests/test_oracle_around.py (finite differences, brute force, hand-worked
blocks, torch's own float8 type).
"""
from __future__ import annotations

import numpy as np

from . import moe

FLT_MAX = float(np.finfo(np.float32).max)
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _f64(a) -> np.ndarray:
    return np.asarray(a, dtype=np.float64)


# -------------------------------------------------------------------- norm
def norm_fwd(S, w, eps):
    S = _f64(S)
    return S / np.sqrt((S * S).mean(axis=1, keepdims=True) + eps) * _f64(w)


def norm_bwd(X, w, dY, dS, eps):
    """dX, dw."""
    X, w, dY = _f64(X), _f64(w), _f64(dY)
    r = 1 / np.sqrt((X * X).mean(axis=1, keepdims=True) + eps)
    dX = r * (dY * w - X * r * r * (dY * w * X).mean(axis=1, keepdims=True))
    if dS is not None:
        dX = dX + _f64(dS)
    return dX, (dY * X * r).sum(axis=0)


# ----------------------------------------------------------------- routing
def masked(logits) -> np.ndarray:
    z = _f64(logits)
    return ~(z > -FLT_MAX)


def scores(logits, score):
    """(p, 1 - p) with p = 0 where masked."""
    z = np.minimum(_f64(logits), FLT_MAX)
    off = masked(logits)
    z = np.where(off, 0.0, z)
    with np.errstate(over="ignore"):
        if score == "sigmoid":
            p, q = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
        else:
            m = np.where(off, -np.inf, z).max(axis=1, keepdims=True)
            e = np.where(off, 0.0, np.exp(z - np.where(np.isfinite(m), m, 0.0)))
            s = e.sum(axis=1, keepdims=True)
            p = np.divide(e, s, out=np.zeros_like(e), where=s > 0)
            q = 1 - p
    return np.where(off, 0.0, p), q


def select(v, k, groups=1, top_groups=1) -> np.ndarray:
    """idx [T, k] of the largest v (-inf: masked), after the groups' choice;
    equal values by the lower id."""
    v = _f64(v)
    T, E = v.shape
    ids = np.arange(E)
    out = np.empty((T, k), dtype=np.int32)
    for t in range(T):
        left = ids
        if groups > 1:
            per = v[t].reshape(groups, -1)
            two = -np.sort(-per, axis=1)[:, :2]
            g = two.sum(axis=1)
            best = sorted(range(groups), key=lambda i: (-g[i], i))[:top_groups]
            left = [e for e in ids if e // per.shape[1] in best]
        out[t] = sorted(left, key=lambda e: (-v[t, e], e))[:k]
    return out


def route_fwd(logits, k, score="softmax", bias=None, groups=1, top_groups=1, renorm=True,
              scale=1.0):
    """(idx, gates)."""
    p, _ = scores(logits, score)
    v = p if bias is None else p + _f64(bias)
    idx = select(np.where(masked(logits), -np.inf, v), k, groups, top_groups)
    return idx, gates_of(p, idx, renorm, scale)


def gates_of(p, idx, renorm, scale):
    g = np.take_along_axis(p, idx.astype(np.int64), axis=1)
    if renorm:
        s = g.sum(axis=1, keepdims=True)
        g = np.divide(g, s, out=np.zeros_like(g), where=s > 0)
    return scale * g


def route_bwd(logits, idx, dgates, score="softmax", renorm=True, scale=1.0):
    """dlogits with the selection held fixed; ids outside [0, E) pass nothing."""
    p, q = scores(logits, score)
    T, E = p.shape
    dz = np.zeros((T, E))
    for t in range(T):
        js = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < E]
        e = np.array([idx[t, j] for j in js], dtype=np.int64)
        dg = scale * _f64(dgates)[t, js]
        g = p[t, e]
        if renorm:
            s = g.sum()
            dg = (dg - (dg * g).sum() / s) / s if s > 0 else 0 * dg
        dp = np.zeros(E)
        np.add.at(dp, e, dg)
        if score == "sigmoid":
            dz[t] = dp * p[t] * q[t]
        elif renorm:
            dz[t] = p[t] * dp     # sum dp p is zero: the gates' sum does not move
        else:
            dz[t] = p[t] * (dp - (dp * p[t]).sum())
    return np.where(masked(logits), 0.0, dz)


# -------------------------------------------------------------- MX formats
def _round_to(v, values):
    """The nearest of the sorted non-negative `values` to |v|, ties to the one
    with an even index (the formats' codes rise with the value), signed."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(values, a, side="left"), 1, len(values) - 1)
    lo = hi - 1
    up, down = values[hi] - a, a - values[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return code, np.copysign(values[code], v)


def e4m3_values() -> np.ndarray:
    """The 127 non-negative finite e4m3 values by code."""
    code = np.arange(127)
    ex, man = code >> 3, code & 7
    return np.where(ex > 0, (8 + man) * 2.0 ** (ex - 10), man * 2.0 ** -9)


def scale_byte(amax, top) -> int:
    """The smallest s >= 0 with amax <= top * 2^(s - 127); 255 if not finite."""
    if not np.isfinite(amax):
        return 255
    s = 0
    while amax > top * 2.0 ** (s - 127):
        s += 1
    return s


def mx_round(x, fmt):
    """Rows x [..., K] in blocks of 32 as "mx8" or "mx4": (codes, scale bytes,
    values); codes carry the sign bit (0x80 or 8)."""
    table, top, sign = (e4m3_values(), 448.0, 0x80) if fmt == "mx8" else (E2M1, 6.0, 8)
    x = _f64(x)
    b = x.reshape(-1, 32)
    s = np.array([scale_byte(a, top) for a in np.abs(b).max(axis=1)])
    f = 2.0 ** (s - 127.0)
    with np.errstate(invalid="ignore"):
        code, val = _round_to(np.where(s[:, None] == 255, 0.0, b / f[:, None]), table)
        val = np.where(s[:, None] == 255, np.nan, val * f[:, None])
    code = np.where(np.signbit(b), code | sign, code).astype(np.uint8)
    return (code.reshape(x.shape), s.reshape(*x.shape[:-1], -1).astype(np.uint8),
            val.reshape(x.shape))


def mx4_row_codes(code) -> np.ndarray:
    """Two codes to a byte, the first in the low half."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def mx4_layout(row_codes, row_scales):
    """Row-major codes [E, N, K/2], scales [E, N, K/32] in the library's order:
    tiles of 16 x 128, lane l = row l % 16, block l / 16."""
    E, N, K2 = row_codes.shape
    K = 2 * K2
    KT, KS = -(-K // 128), -(-K // 512)
    c = np.zeros((E, N, KT * 64), np.uint8)
    c[:, :, :K2] = row_codes
    s = np.full((E, N, KS * 16), 127, np.uint8)
    s[:, :, :K // 32] = row_scales
    # [E, NT, 16, KT, 4, 16] -> [E, NT, KT, 4, 16, 16]
    c = c.reshape(E, N // 16, 16, KT, 4, 16).transpose(0, 1, 3, 4, 2, 5)
    # [E, NT, 16, KS, 4 tiles, 4 blocks] -> [E, NT, KS, 4 blocks, 16, 4 tiles]
    s = s.reshape(E, N // 16, 16, KS, 4, 4).transpose(0, 1, 3, 5, 2, 4)
    return c.reshape(E, -1), s.reshape(E, -1)


# ------------------------------------------------------------ MX4 experts
def moe_fwd_mx(X, idx, gates, W1, W2, mx8: bool):
    """Y of the layer with given weight values; with `mx8` the SwiGLU output is
    rounded to MX8 before the second product."""
    X, W1, W2, gates = _f64(X), _f64(W1), _f64(W2), _f64(gates)
    if not mx8:
        return moe.moe_fwd(X, idx, gates, W1, W2, 1)
    E, F = W1.shape[0], W2.shape[2]
    Y = np.zeros((X.shape[0], W2.shape[1]))
    for e in range(E):
        t, j = np.nonzero(np.asarray(idx) == e)
        if t.size == 0:
            continue
        u = X[t] @ W1[e].T
        with np.errstate(over="ignore"):
            a = u[:, :F] / (1 + np.exp(-u[:, :F])) * u[:, F:]
        y = mx_round(a, "mx8")[2] @ W2[e].T
        np.add.at(Y, t, gates[t, j][:, None] * y)
    return Y
