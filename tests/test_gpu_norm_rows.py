"""The norm's gradient where a workgroup takes several rows, in every variant
(one, two and four vectors a lane, up to 512 and 1024 threads), and the norm
written over its inputs.  Oracle and tolerances of test_gpu_norm_route.py."""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from test_gpu_norm_route import EPS, draw, f64, gen, mf, nan_out  # noqa: F401

pytestmark = pytest.mark.gpu

ROWS = [("bf16", 8200, 64), ("bf16", 8200, 512), ("bf16", 1700, 1088), ("bf16", 700, 7168),
        ("bf16", 700, 8256), ("bf16", 700, 16384), ("f32", 8200, 64), ("f32", 8200, 256),
        ("f32", 1100, 4160), ("f32", 700, 8192), ("f32", 700, 8256), ("f32", 700, 16384)]


@pytest.mark.parametrize("dtype,T,h", ROWS)
def test_gradient_over_several_rows(mf, dtype, T, h):
    t = torch()
    g = gen(T + h)
    X, w, dY, dS = (draw(g, *s, dtype=dtype) for s in ((T, h), (h,), (T, h), (T, h)))
    Xd, wd, dYd, dSd = (a.cuda() for a in (X, w, dY, dS))
    x, ww, dy = f64(X), f64(w), f64(dY)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    r = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + EPS)
    mag = r * (np.abs(dy * ww) + np.abs(x) * r * r * np.abs(dy * ww * x).mean(axis=1, keepdims=True))
    mag_w = np.abs(dy * x * r).sum(axis=0)
    tol_w = ((T + 20) * 2.0 ** -24 + 2e-6) * mag_w
    for residual in (False, True):
        log("norm backward", dtype, T, h, residual)
        dX, dw = nan_out((T, h), X), t.full((h,), float("nan"), device="cuda")
        mf.memfine_norm_bwd(EPS, Xd, wd, dYd, dX, dw, dS=dSd if residual else None)
        rX, rw = oa.norm_bwd(x, ww, dy, f64(dS) if residual else None, EPS)
        m = mag + np.abs(f64(dS)) if residual else mag
        assert np.all(np.abs(f64(dX) - rX) <= (half + 1e-5) * m)
        assert np.all(np.abs(f64(dw) - rw) <= tol_w)
    # over each of the gradients that come in: the same bits
    for over in (dYd, dSd):
        ins = [dYd.clone(), dSd.clone()]
        out = ins[0] if over is dYd else ins[1]
        again = t.full((h,), float("nan"), device="cuda")
        mf.memfine_norm_bwd(EPS, Xd, wd, ins[0], out, again, dS=ins[1])
        assert t.equal(out, dX) and t.equal(again, dw)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,h", [(9, 64), (5, 1088), (7, 7168), (3, 8256), (3, 16384)])
def test_norm_over_its_inputs(mf, T, h, dtype):
    """S may be X or R."""
    t = torch()
    g = gen(T * h)
    X, R, w = (draw(g, *s, dtype=dtype).cuda() for s in ((T, h), (T, h), (h,)))
    S, Y = nan_out((T, h), X), nan_out((T, h), X)
    mf.memfine_norm_fwd(EPS, X, w, R=R, S=S, Y=Y)
    for over in (0, 1):
        ins = [X.clone(), R.clone()]
        Y2 = nan_out((T, h), X)
        mf.memfine_norm_fwd(EPS, ins[0], w, R=ins[1], S=ins[over], Y=Y2)
        assert t.equal(ins[over], S) and t.equal(Y2, Y)
