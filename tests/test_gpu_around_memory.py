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


def test_captured_calls_keep_their_memory(mf):
    """Calls without an allocator that were captured into a graph: replays give the
    eager results whatever the capture's stream does in between (larger calls,
    which replace its block, trimming) and beside work on other streams."""
    t = torch()
    rng = np.random.default_rng(11)
    bf = t.bfloat16
    T, N, K, h, F, E, k = 16, 528, 8224, 256, 320, 6, 2   # K over 4096: split and summed
    lin = packed(mf, 1, N, K, *rows(rng, 1, N, K)[:2])
    w1 = packed(mf, E, 2 * F, h, *rows(rng, E, 2 * F, h, 119, 122)[:2])
    w2 = packed(mf, E, h, F, *rows(rng, E, h, F, 119, 122)[:2])
    big = packed(mf, 1, 1040, 12320, *rows(rng, 1, 1040, 12320)[:2])
    shape = mf.make_shape(T, h, F, E, k, mf.BF16)
    w, Wr = t.randn(h, device="cuda").to(bf), t.randn(E, h, device="cuda").to(bf)
    wide = t.randn(64, 12320, device="cuda").to(bf)
    idx = dev(rng.integers(0, E, (T, k)).astype(np.int32))
    g = t.rand(T, k, device="cuda")
    X, R, dl = t.empty(T, K, dtype=bf, device="cuda"), t.empty(T, h, dtype=bf, device="cuda"), t.empty(T, E, device="cuda")

    def results():
        return [t.zeros(T, N, device="cuda"), t.zeros(T, h, dtype=bf, device="cuda"),
                t.zeros(T, h, dtype=bf, device="cuda"), t.zeros(h, device="cuda"),
                t.zeros(T, h, dtype=bf, device="cuda"), t.zeros(E, h, device="cuda")]

    def calls(o):
        mf.memfine_linear_mxw(N, K, X, *lin, o[0])
        mf.memfine_moe_fwd_mxw(shape, 2, R, idx, g, *w1, *w2, o[1])
        mf.memfine_norm_bwd(1e-6, R, w, R, o[2], o[3])
        mf.memfine_router_logits_bwd(shape, R, Wr, dl, o[4], o[5])

    def other(n):
        out = t.empty(64, 1040, device="cuda")
        for _ in range(n):
            mf.memfine_linear_mxw(1040, 12320, wide, *big, out)
        return out

    side, third = t.cuda.Stream(), t.cuda.Stream()
    want_other = other(1)
    graphs, outs = [], []
    for _ in range(2):
        t.cuda.synchronize()
        with t.cuda.stream(side):
            mf.memfine_workspace_trim(0)
        log("capture")
        graph, o = t.cuda.CUDAGraph(), results()
        with t.cuda.graph(graph, stream=side):
            calls(o)
        with t.cuda.stream(side):
            assert mf.memfine_workspace_held() == 0
        graphs.append(graph)
        outs.append(o)
    for i in range(6):
        X.copy_(t.randn(X.shape, device="cuda"))
        R.copy_(t.randn(R.shape, device="cuda"))
        dl.copy_(t.randn(dl.shape, device="cuda"))
        want = results()
        calls(want)
        t.cuda.synchronize()
        log("replay", i)
        with t.cuda.stream(side):
            if i == 4:
                mf.memfine_workspace_trim(0)
            got_other = other(20)
        with t.cuda.stream(third):
            graphs[i % 2].replay()          # beside work on the stream that it was captured on
        with t.cuda.stream(side):
            graphs[1 - i % 2].replay()
        t.cuda.synchronize()
        assert t.equal(got_other, want_other), i
        for o in outs:
            assert all(t.equal(a, b) for a, b in zip(o, want)), i
            for x in o:
                x.zero_()


@pytest.mark.parametrize("mx8", (False, True))
def test_linear_on_the_callers_memory(mf, mx8):
    """A split reduction takes the documented bytes from the caller's allocator
    and gives them back; a failing allocator is an error that leaves nothing."""
    from test_gpu_mxw import activations
    t = torch()
    rng = np.random.default_rng(12)
    for T, N, K in ((16, 528, 8224), (64, 96, 4128), (16, 96, 4096), (1, 96, 8192)):
        W = packed(mf, 1, N, K, *rows(rng, 1, N, K)[:2])
        X, XS, _ = activations(rng, T, K, mx8)
        want, got = (t.full((T, N), float("nan"), device="cuda") for _ in range(2))
        mf.memfine_linear_mxw(N, K, X, *W, want, XS=XS)
        a, need = mf.TorchAllocator(), mf.memfine_linear_mxw_workspace_bytes(T, N, K, mx8)
        side = t.cuda.Stream()
        t.cuda.synchronize()
        with t.cuda.stream(side):
            mf.memfine_workspace_trim(0)
            mf.memfine_linear_mxw(N, K, X, *W, got, XS=XS, allocator=a)
            assert mf.memfine_workspace_held() == 0
        side.synchronize()
        assert t.equal(got, want)
        assert (a.high_water, a.calls, a.live_bytes) == (need, int(need > 0), 0)
        a = mf.TorchAllocator()
        a.fail_at = 1
        if need:
            with pytest.raises(mf.MemfineError) as e:
                mf.memfine_linear_mxw(N, K, X, *W, got, XS=XS, allocator=a)
            assert e.value.code == -4 and a.live_bytes == 0
