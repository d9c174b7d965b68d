"""Memory of the calls around the layer: where it comes from, in which stream's
order, and what of it a captured graph keeps."""
import numpy as np
import pytest

from gpu_harness import log, torch
from test_gpu_mxw import dev, f64, mf, packed, rows  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pack", (False, True))
def test_matrices_made_in_the_order_of_the_calls_stream(mf, pack):
    """Memory that the current stream has just given back may still be in use on
    it: a call on another stream does not take it for its results."""
    t = torch()
    E, N, K = 3, 4096, 4096
    W = t.randn((E, N, K), device="cuda").to(t.bfloat16)
    want = mf.memfine_mxw_quantize(W)
    rc = t.zeros((E, N, K // 2), dtype=t.uint8, device="cuda")
    rs = t.full((E, N, K // 32), 127, dtype=t.uint8, device="cuda")
    side = t.cuda.Stream()
    t.cuda.synchronize()
    given_back = [t.empty_like(x) for x in want]
    at = {x.data_ptr() for x in given_back}
    del given_back
    log(f"results on a side stream, pack={pack}")
    got = (mf.memfine_mxw_pack(E, N, K, rc, rs, stream=side) if pack
           else mf.memfine_mxw_quantize(W, stream=side))
    side.synchronize()
    assert not at & {x.data_ptr() for x in got}
    if pack:
        assert t.all(got[0] == 0) and t.all(got[1] == 127)
    else:
        assert all(t.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("E", (1, 8, 33, 64, 65, 128, 160, 200, 256))
def test_router_logits_take_no_memory(mf, E, dtype):
    """The same logits as the router's own, and nothing from the stream's block."""
    t = torch()
    side = t.cuda.Stream()
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    T, h = 77, 448
    shape = mf.make_shape(T, h, 64, E, 1, mf.BF16 if dtype == "bf16" else mf.F32)
    X, Wr = t.randn(T, h, device="cuda").to(dt), t.randn(E, h, device="cuda").to(dt)
    z, want = (t.full((T, E), float("nan"), device="cuda") for _ in range(2))
    idx, gates = t.zeros((T, 1), dtype=t.int32, device="cuda"), t.zeros((T, 1), device="cuda")
    mf.memfine_router_fwd(shape, X, Wr, idx, gates, want)
    t.cuda.synchronize()
    log(f"router logits E={E} {dtype}")
    with t.cuda.stream(side):
        mf.memfine_workspace_trim(0)
        mf.memfine_router_logits(shape, X, Wr, z)
        assert mf.memfine_workspace_held() == 0
    side.synchronize()
    assert t.equal(z, want)
