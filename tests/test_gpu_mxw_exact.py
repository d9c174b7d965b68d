"""MX4 products whose sums are exact whatever their order: a block of the
reduction that is lost, or taken twice, shows in one output.

Activations 0, +-1, +-2, +-3 (exact in bf16 and in e4m3) and every e2m1 value, all
scales 1: products are multiples of 0.5 of at most 18, so the matrix core's cut
at 2^-13 of the largest of eight takes nothing, and sums of up to 2^18 of them are
exact floats."""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from test_gpu_mxw import LINEAR, dev, f64, mf  # noqa: F401
from test_gpu_mxw_kernels import SPLIT

pytestmark = pytest.mark.gpu

MANY = [(2049, 4112, 544), (4097, 16400, 160)]


@pytest.mark.parametrize("mx8", (False, True))
@pytest.mark.parametrize("T,N,K", LINEAR + SPLIT + MANY)
def test_linear_exact(mf, T, N, K, mx8):
    t = torch()
    rng = np.random.default_rng(T + N + K)
    code = rng.integers(0, 16, (N, K)).astype(np.uint8)
    W = mf.memfine_mxw_pack(1, N, K, dev(oa.mx4_row_codes(code)[None]),
                            t.full((1, N, K // 32), 127, dtype=t.uint8, device="cuda"))
    x = rng.integers(-3, 4, (T, K))
    X, XS = t.from_numpy(x.astype(np.float32)).to(t.bfloat16).cuda(), None
    if mx8:  # e4m3: 1 is 0x38, 2 0x40, 3 0x44
        X = dev(np.array([0, 0x38, 0x40, 0x44], np.uint8)[np.abs(x)] | np.where(x < 0, 0x80, 0).astype(np.uint8))
        XS = t.full((T, K // 32), 127, dtype=t.uint8, device="cuda")
    log("exact", T, N, K, mx8)
    Y = t.full((T, N), float("nan"), device="cuda")
    mf.memfine_linear_mxw(N, K, X, *W, Y, XS=XS)
    w = np.where(code >= 8, -1.0, 1.0) * oa.E2M1[code & 7]
    pick = np.unique(np.concatenate([rng.integers(0, T, 80), np.arange(min(T, 70)), [T - 1]]))
    assert np.array_equal(f64(Y[t.from_numpy(pick).cuda()]), x[pick].astype(np.float64) @ w.T)
