"""The attention's calls on tensors beyond 4 GiB, on scale bytes at their ends, on
padded batches, and beside each other on streams and in graphs."""
import numpy as np
import pytest

from gpu_harness import log, torch
from test_gpu_attn import Case, mf  # noqa: F401
from test_gpu_cache import Pages, check_decode, f64, gen, ints, offsets_of, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_rows_beyond_4_gib(mf, dtype):  # noqa: F811
    """Rows far apart: the last ones lie past 2^32 bytes of queries, keys and values, and
    of their gradients."""
    t = torch()
    c = Case(mf, [130, 0, 77], 4, 2, 64, dtype, before=40000, after=3)
    small = Case(mf, [130, 0, 77], 4, 2, 64, dtype)
    c.x[40000:-3], c.do[40000:-3] = small.x, small.do
    c.upload()
    want = small.forward()
    ld = 57344 if dtype == "bf16" else 28672
    wide = t.zeros(c.T, ld, dtype=c.dev.dtype, device="cuda")
    assert 40000 * ld * wide.element_size() > 2 ** 32
    at = ld - c.dev[0].numel()
    rows = wide[:, at:].unflatten(1, c.dev.shape[1:])
    rows.copy_(c.dev)
    c.dev = rows
    log(f"rows of {ld} {dtype}")
    O, lse = c.forward()
    keep = slice(40000, c.T - 3)
    assert t.equal(O[keep], want[0]) and t.equal(lse[:, keep], want[1])
    d = t.full_like(wide, float("nan"))
    drows = d[:, at:].unflatten(1, c.dev.shape[1:])
    mf.memfine_attn_bwd(c.attn, c.offsets, *c.split(c.dev), O, lse, c.ddo, *c.split(drows))
    c.check_backward(O, lse, drows)   # (sums of the heads' parts: not the same bits)
    assert t.all(t.isnan(d[keep, :at]))
    # and the rotation, in place
    cos, sin = (y.cuda() for y in tables(130, 64))
    Y = t.empty_like(small.dev)
    mf.memfine_rope(small.offsets, cos, sin, small.dev, Y)
    mf.memfine_rope(c.offsets, cos, sin, rows, rows)
    assert t.equal(rows[keep], Y)


@pytest.mark.parametrize("held", ("bf16", "mx8"))
def test_cache_beyond_4_gib(mf, held):  # noqa: F811
    """Pages past 2^32 bytes of keys are written and read like others."""
    t = torch()
    Hk, D, page, pages = 8, 128, 64, 33000 if held == "bf16" else 66000
    lens, H = [700, 65, 1], 16
    p = Pages(mf, lens, Hk, D, page, held)
    one = 2 if held == "bf16" else 1
    size = (pages, Hk, page, D)
    big = [t.zeros(size, dtype=p.dev[0].dtype, device="cuda") for _ in range(2)]
    assert big[0].numel() * one > 2 ** 32
    sc = [None if held == "bf16" else t.zeros((*size[:3], D // 32), dtype=t.uint8, device="cuda")
          for _ in range(2)]
    cache = mf.make_cache(*big, *sc)
    shift = pages - p.pages
    table = t.where(p.dtable >= 0, p.dtable + shift, p.dtable).contiguous()
    x = t.randn(sum(lens), H + 2 * Hk, D, generator=gen(3)).to(t.bfloat16).cuda()
    off, n = ints(offsets_of(lens)), ints(lens)
    R = t.empty(sum(lens), H, D, dtype=t.bfloat16, device="cuda")
    log(f"cache of {big[0].numel() * one >> 30} GiB, {held}")
    for c, tab in ((p.cache, p.dtable), (cache, table)):
        mf.memfine_kv_write(c, tab, n, x[:, H:H + Hk], x[:, H + Hk:], offsets=off, Q=x[:, :H], R=R)
    used = sorted(set(table[table >= 0].tolist()))
    for i in range(2):
        assert t.equal(big[i][used][:, :, :1], p.dev[i][[u - shift for u in used]][:, :, :1])
    q = x[off[1:].long() - 1, :H]
    outs = [t.empty(3, H, D, dtype=t.bfloat16, device="cuda") for _ in range(2)]
    attn = mf.make_attn(H, Hk, D)
    mf.memfine_attn_decode(attn, p.cache, p.dtable, n, q, outs[0])
    mf.memfine_attn_decode(attn, cache, table, n, q, outs[1])
    assert t.equal(outs[0], outs[1])
    check_decode(mf, p, lens, H, q=t.cat([q, q[:, :1]], 1).cpu())


def test_scale_bytes_at_their_ends(mf):  # noqa: F811
    """Scale 255 makes a block NaN whatever its codes are: in keys the token's weights, so
    the whole output, in values the block's columns.  Scale 0 is 2^-127."""
    t = torch()
    lens = [40, 40, 40, 40]
    p = Pages(mf, lens, 1, 64, 16, "mx8")
    for i in range(4):
        which, byte = i & 1, 255 if i < 2 else 0
        page = p.table[i, 1]
        p.sdev[which][page, 0, 3, 1] = byte       # token 19, columns 32 to 63
        p.dev[which][page, 0, 3, 32:] = 0 if i < 2 else 0x7e
        p.scales[which], p.kv[which] = p.sdev[which].cpu(), p.dev[which].cpu()
    attn = mf.make_attn(2, 1, 64)
    q = t.randn(4, 2, 64, generator=gen(1)).to(t.bfloat16).cuda()
    O = t.zeros_like(q)
    log("scale bytes 255 and 0")
    mf.memfine_attn_decode(attn, p.cache, p.dtable, ints(lens), q, O)
    assert t.all(t.isnan(O[0]))
    assert t.all(t.isnan(O[1, :, 32:])) and t.all(t.isfinite(O[1, :, :32]))
    assert t.all(t.isfinite(O[2:]))
    # the last two as if the token's block were zeros, to 448 2^-127
    for i in (2, 3):
        p.dev[i & 1][p.table[i, 1], 0, 3, 32:] = 0
    Z = t.zeros_like(O)
    mf.memfine_attn_decode(attn, p.cache, p.dtable, ints(lens), q, Z)
    assert t.equal(Z[2:], O[2:])


def test_written_rows_that_are_not_finite(mf):  # noqa: F811
    """A NaN or an infinity in a new key or value makes its own block NaN in MX8 and stays
    itself in bf16."""
    t = torch()
    for held in ("bf16", "mx8"):
        p = Pages(mf, [16], 2, 64, 16, held)
        x = t.randn(16, 4, 64, generator=gen(2)).to(t.bfloat16)
        x[3, 0, 5], x[4, 3, 40] = float("nan"), float("inf")
        dev = x.cuda()
        log(f"rows that are not finite, {held}")
        mf.memfine_kv_write(p.cache, p.dtable, ints([16]), dev[:, :2], dev[:, 2:], offsets=ints([0, 16]))
        k, v = (p.values(i)[p.table[0, 0]].swapaxes(0, 1) for i in range(2))
        bad_k, bad_v = ~np.isfinite(k), ~np.isfinite(v)
        where_k, where_v = np.zeros_like(bad_k), np.zeros_like(bad_v)
        if held == "bf16":
            where_k[3, 0, 5], where_v[4, 1, 40] = True, True
        else:
            where_k[3, 0, :32], where_v[4, 1, 32:] = True, True
        assert np.array_equal(bad_k, where_k) and np.array_equal(bad_v, where_v)


def test_padded_batch(mf):  # noqa: F811
    """Places without a sequence: length 0, no pages, whatever their rows hold."""
    t = torch()
    lens = [50, 0, 129, 0]
    p = Pages(mf, lens, 2, 128, 32, "bf16")
    q = t.randn(4, 5, 128, generator=gen(6)).to(t.bfloat16)
    q[[1, 3]] = float("nan")
    log("padded batch")
    O, lse, _, _ = check_decode(mf, p, lens, 4, q=q)
    assert t.all(O[[1, 3]] == 0) and t.all(lse[[1, 3]] == -float("inf"))
    p = Pages(mf, [0, 0], 2, 128, 32, "bf16")
    O, _, _, _ = check_decode(mf, p, [0, 0], 4)
    assert t.all(O == 0)


def test_calls_beside_each_other(mf):  # noqa: F811
    """Calls without an allocator on two streams, and two graphs captured on one stream,
    keep apart what they work in."""
    t = torch()
    jobs = []
    for seed, (lens, held) in enumerate((([9000, 40], "bf16"), ([300, 7000, 2500], "mx8"))):
        p = Pages(mf, lens, 2, 128, 64, held, seed=seed)
        q = (t.randn(len(lens), 8, 128, generator=gen(seed))).to(t.bfloat16).cuda()
        c = Case(mf, [1500 + 300 * seed], 32, 2, 64, "bf16", seed=seed)
        O, lse = c.forward()
        jobs.append((p, ints(lens), q, c, O, lse))

    def call(job, out, d):
        p, n, q, c, O, lse = job
        mf.memfine_attn_decode(mf.make_attn(8, 2, 128), p.cache, p.dtable, n, q, out)
        mf.memfine_attn_bwd(c.attn, c.offsets, *c.split(c.dev), O, lse, c.ddo, *c.split(d))
    want = []
    for j in jobs:
        out, d = t.zeros_like(j[2]), t.zeros_like(j[3].dev)
        call(j, out, d)
        want.append((out, d))
    streams = [t.cuda.Stream() for _ in jobs]
    got = [(t.zeros_like(o), t.zeros_like(d)) for o, d in want]
    t.cuda.synchronize()
    log("two streams")
    for _ in range(4):
        for j, s, g in zip(jobs, streams, got):
            with t.cuda.stream(s):
                call(j, *g)
    t.cuda.synchronize()
    assert all(t.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))
    graphs = []
    for j, g in zip(jobs, got):
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph, stream=streams[0]):
            call(j, *g)
        graphs.append(graph)
    for i in range(3):
        log(f"replays {i}")
        for g in got:
            for x in g:
                x.zero_()
        t.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with t.cuda.stream(s):
                graph.replay()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))
