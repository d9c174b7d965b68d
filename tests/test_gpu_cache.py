"""GPU parity of the rotation, of the cache's writes and of the attention over the cache
against oracle/attention.py, which starts from the same stored inputs in float64.

Tolerances, from the arithmetic (u = 2^-24):
* a turned value: two products and a sum, 3 u of |x_a c| + |x_b s|, and half a
  step of bf16, 2^-8 of the value.
* in MX8: that, and half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below
  the normals), with the block's own scale unless its maximum lies within
  1e-5 of the scale's limit.  Values that are not turned: the same bits.
* O over the cache: as over packed sequences (tests/test_gpu_attn.py), with weights
  rounded to bf16; the cached values are exact in bf16.
"""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from oracle import attention as at

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B = 2.0 ** -8


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


def gen(seed):
    return torch().Generator().manual_seed(int(seed))


def ints(x):
    return torch().tensor(np.asarray(x), dtype=torch().int32, device="cuda")


def tables(n, D):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    t = torch()
    return t.from_numpy(np.cos(a)).float(), t.from_numpy(np.sin(a)).float()


def offsets_of(lens, before=0):
    return before + np.concatenate([[0], np.cumsum(lens)])


# ---------------------------------------------------------------- rotation
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("lens,H", [([1], 1), ([3, 0, 40], 5), ([17, 200], 33), ([2] * 130, 4)],
                         ids=("one", "three", "two", "many"))
def test_rope(mf, lens, H, D, interleaved, dtype):
    t = torch()
    log(f"rope {len(lens)} sequences, {H} heads of {D}, {dtype}")
    off = offsets_of(lens, 2)
    T = off[-1] + 3
    dt = t.bfloat16 if dtype == "bf16" else t.float32
    x = t.randn(T, H + 2, D, generator=gen(T)).to(dt)   # heads of a wider row
    cos, sin = tables(max(lens), D)
    dev, o = x.cuda(), ints(off)
    Y = t.full((T, H, D), float("nan"), dtype=dt, device="cuda")
    pos = np.concatenate([np.arange(n) for n in lens])
    rows = slice(2, off[-1])
    half = B if dtype == "bf16" else U
    for inverse in (False, True):
        Y.fill_(float("nan"))
        mf.memfine_rope(o, cos.cuda(), sin.cuda(), dev[:, 1:H + 1], Y, interleaved=interleaved,
                        inverse=inverse)
        ref, mag = at.rope(f64(x)[rows, 1:H + 1], f64(cos)[pos], f64(sin)[pos], interleaved, inverse)
        got = f64(Y)
        assert np.all(np.abs(got[rows] - ref) <= half * np.abs(ref) + 3 * U * mag)
        assert np.all(np.isnan(got[:2])) and np.all(np.isnan(got[off[-1]:]))
    # in place, in the wider row
    keep = dev.clone()
    mf.memfine_rope(o, cos.cuda(), sin.cuda(), dev[:, 1:H + 1], dev[:, 1:H + 1],
                    interleaved=interleaved, inverse=True)
    assert t.equal(dev[rows, 1:H + 1], Y[rows])
    assert t.equal(dev[:, 0], keep[:, 0]) and t.equal(dev[:, -1], keep[:, -1])
    assert t.equal(dev[:2], keep[:2]) and t.equal(dev[off[-1]:], keep[off[-1]:])


def test_rope_past_the_tables(mf):
    t = torch()
    cos, sin = tables(5, 64)
    X = t.randn(9, 3, 64, generator=gen(1)).cuda()
    Y = t.zeros_like(X)
    mf.memfine_rope(ints([0, 2, 9]), cos.cuda(), sin.cuda(), X, Y)
    bad = [7, 8]
    assert t.all(t.isnan(Y[bad])) and t.all(t.isfinite(Y[:7]))


# -------------------------------------------------------------------- cache
class Pages:
    """A cache with a shuffled table, its pages full of `fill`."""

    def __init__(self, mf, need, Hk, D, page, held, seed=0, fill=None, spare=2, width=None):
        t = torch()
        rng = np.random.default_rng(seed)
        count = [-(-n // page) for n in need]
        self.pages, self.width = sum(count) + spare, width or max(count + [1])
        self.page, self.Hk, self.D, self.held = page, Hk, D, held
        order, self.table = rng.permutation(self.pages), np.full((len(need), self.width), -1)
        at_ = 0
        for b, c in enumerate(count):
            self.table[b, :c] = order[at_:at_ + c]
            at_ += c
        size = (self.pages, Hk, page, D)
        g = gen(seed + 5)
        self.kv, self.scales = [], [None, None]
        for i in range(2):
            if held == "bf16":
                x = t.randn(size, generator=g).to(t.bfloat16)
                self.kv.append(x if fill is None else t.full_like(x, fill))
            elif fill is not None:
                self.kv.append(t.full(size, 0x7f, dtype=t.uint8))
                self.scales[i] = t.full((*size[:3], D // 32), 255, dtype=t.uint8)
            else:
                code = rng.integers(0, 0x77, size) | rng.integers(0, 2, size) << 7
                self.kv.append(t.from_numpy(code.astype(np.uint8)))
                self.scales[i] = t.from_numpy(rng.integers(118, 122, (*size[:3], D // 32)).astype(np.uint8))
        self.dev = [x.cuda() for x in self.kv]
        self.sdev = [None if x is None else x.cuda() for x in self.scales]
        self.cache = mf.make_cache(*self.dev, *self.sdev)
        self.dtable = ints(self.table)

    def values(self, i, dev=True):
        """float64 [pages, kv_heads, page, D] of keys (0) or values (1)."""
        x = (self.dev if dev else self.kv)[i]
        if self.held == "bf16":
            return f64(x)
        code = x.cpu().numpy()
        v = np.concatenate([oa.e4m3_values(), [np.nan]])[code & 0x7f] * np.where(code & 0x80, -1, 1)
        s = (self.sdev if dev else self.scales)[i].cpu().numpy()
        return v * np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127)).repeat(32, -1)

    def tokens(self, i, b, n):
        """[n, kv_heads, D] of sequence b; tokens without a page are left out."""
        t = np.arange(n)
        ids = self.table[b, t // self.page]
        ok = (ids >= 0) & (ids < self.pages)
        return self.values(i)[ids[ok], :, t[ok] % self.page]


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("turned", (None, False, True), ids=("plain", "halves", "interleaved"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("lens,past,page,H,Hk", [([1], [0], 16, 1, 1), ([1, 1, 1], [0, 15, 300], 16, 8, 2),
                                                 ([5, 0, 70], [3, 9, 0], 32, 7, 7),
                                                 ([33, 1], [64, 1], 64, 40, 9)], ids=str)
def test_write(mf, lens, past, page, H, Hk, D, turned, held):
    t = torch()
    log(f"write {lens} after {past}, pages of {page}, {held}, turned {turned}")
    ends = [a + b for a, b in zip(lens, past)]
    p = Pages(mf, ends, Hk, D, page, held)
    before = [p.values(i) for i in range(2)]
    T = sum(lens)
    x = t.randn(T, H + 2 * Hk, D, generator=gen(T + D)).to(t.bfloat16)
    dev = x.cuda()
    Q, K, V = dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:]
    R = t.full((T, H, D), float("nan"), dtype=t.bfloat16, device="cuda")
    cos, sin = tables(max(ends), D)
    kw = {} if turned is None else dict(cos=cos.cuda(), sin=sin.cuda(), interleaved=turned)
    one = all(n == 1 for n in lens)
    off = ints(offsets_of(lens))
    mf.memfine_kv_write(p.cache, p.dtable, ints(ends), K, V, offsets=None if one else off, Q=Q, R=R, **kw)
    pos = np.concatenate([np.arange(a, a + n) for n, a in zip(lens, past)])
    seq = np.repeat(np.arange(len(lens)), lens)

    def want(y):
        if turned is None:
            return f64(y), np.zeros(y.shape)
        return at.rope(f64(y), f64(cos)[pos], f64(sin)[pos], turned)
    ref, mag = want(x[:, :H])
    exact = turned is None
    assert np.all(np.abs(f64(R) - ref) <= (0 if exact else B * np.abs(ref) + 3 * U * mag))
    new = [want(x[:, H:H + Hk]), (f64(x[:, H + Hk:]), 0)]
    for i in range(2):
        got, same = p.values(i), np.ones((p.pages, page), bool)
        where = (p.table[seq, pos // page], pos % page)
        same[where] = False
        old = np.moveaxis(before[i], 2, 1)
        assert np.array_equal(np.moveaxis(got, 2, 1)[same], old[same])   # nothing else changed
        got = got[where[0], :, where[1]]
        ref, mag = new[i]
        if held == "bf16":
            tol = 0 if i or exact else B * np.abs(ref) + 3 * U * mag
            assert np.all(np.abs(got - ref) <= tol)
            continue
        if i or exact:
            assert np.array_equal(got, oa.mx_round(ref, "mx8")[2])
            continue
        s = f64(p.sdev[i])[where[0], :, where[1]]
        top, lim = np.abs(ref).reshape(*s.shape, 32).max(-1), 448 * 2.0 ** (s - 127)
        assert np.all((top <= lim * (1 + 1e-5)) & (top > lim / 2 * (1 - 1e-5)))
        step = np.maximum(np.abs(ref) * 2.0 ** -4, (2.0 ** (s - 137)).repeat(32, -1))
        assert np.all(np.abs(got - ref) <= (1 + 1e-4) * step + 3 * U * mag)
    # again without queries: the same
    held_now = [d.clone() for d in p.dev]
    mf.memfine_kv_write(p.cache, p.dtable, ints(ends), K, V, offsets=off, **kw)
    assert all(t.equal(a, b) for a, b in zip(held_now, p.dev))


def test_write_without_a_place(mf):
    """Padded rows, tokens before the first, past the table's width, and entries that
    are no page: nothing is written for them, queries of dropped rows are left."""
    t = torch()
    p = Pages(mf, [32, 32, 32, 32], 2, 64, 16, "bf16", spare=0)
    p.table[1, 0], p.table[2, 1] = -1, p.pages
    p.dtable = ints(p.table)
    before = [d.clone() for d in p.dev]
    lengths = ints([0, 5, 20, 40])      # none; no page; no page; past the width
    x = t.randn(4, 8, 64, generator=gen(2)).to(t.bfloat16).cuda()
    R = t.full((4, 4, 64), 7.0, dtype=t.bfloat16, device="cuda")
    log("writes without a place")
    mf.memfine_kv_write(p.cache, p.dtable, lengths, x[:, 4:6], x[:, 6:], Q=x[:, :4], R=R)
    assert all(t.equal(a, b) for a, b in zip(before, p.dev))
    assert t.all(R[[0, 3]] == 7) and t.equal(R[[1, 2]], x[[1, 2], :4])
    # more rows than tokens: the first ones are dropped
    mf.memfine_kv_write(p.cache, p.dtable, ints([2, 0, 0, 0]), x[:, 4:6], x[:, 6:],
                        offsets=ints([0, 4, 4, 4, 4]))
    page = p.dev[0][p.table[0, 0]]
    assert t.equal(page[:, 0], x[2, 4:6]) and t.equal(page[:, 1], x[3, 4:6])
    assert t.equal(page[:, 2:], before[0][p.table[0, 0]][:, 2:])
    # a position past the tables is NaN, in the cache too
    cos, sin = (y.cuda() for y in tables(1, 64))
    mf.memfine_kv_write(p.cache, p.dtable, ints([2, 0, 0, 0]), x[:, 4:6], x[:, 6:],
                        offsets=ints([0, 1, 1, 1, 1]), cos=cos, sin=sin)
    assert t.all(t.isnan(p.dev[0][p.table[0, 0]][:, 1]))
    assert t.equal(p.dev[1][p.table[0, 0]][:, 1], x[0, 6:])


def test_write_queries_in_place(mf):
    t = torch()
    p = Pages(mf, [20], 2, 128, 32, "mx8")
    x = t.randn(20, 4, 128, generator=gen(4)).to(t.bfloat16).cuda()
    kv = t.randn(20, 2, 128, generator=gen(5)).to(t.bfloat16).cuda()
    cos, sin = (y.cuda() for y in tables(20, 128))
    R = t.empty_like(x)
    kw = dict(offsets=ints([0, 20]), cos=cos, sin=sin)
    mf.memfine_kv_write(p.cache, p.dtable, ints([20]), kv, kv, Q=x, R=R, **kw)
    mf.memfine_kv_write(p.cache, p.dtable, ints([20]), kv, kv, Q=x, R=x, **kw)
    assert t.equal(x, R)


# ------------------------------------------------------------------- decode
def check_decode(mf, p, lens, H, window=0, seed=0, tokens=None, q=None, want_lse=True):
    t = torch()
    D, n = p.D, len(lens)
    attn = mf.make_attn(H, p.Hk, D, window=window)
    if q is None:
        q = (t.randn(n, H + 1, D, generator=gen(seed)) * 1.5).to(t.bfloat16)
    dev = q.cuda()
    O = t.full((n, H, D), float("nan"), dtype=t.bfloat16, device="cuda")
    lse = t.full((n, H), float("nan"), device="cuda")
    mf.memfine_attn_decode(attn, p.cache, p.dtable, ints(lens), dev[:, :H], O, lse if want_lse else None)
    got, gl = f64(O), f64(lse)
    k, v = p.values(0), p.values(1)
    for b, m in enumerate(lens):
        s = np.arange(min(m, p.width * p.page))
        if window:
            s = s[max(0, len(s) - window):]
        ids = p.table[b, s // p.page]
        ok = (ids >= 0) & (ids < p.pages)
        kk, vv = (x[ids[ok], :, s[ok] % p.page] for x in (k, v))
        ref, rl, A, big = at.decode(f64(q)[b, :H], kk, vv, D ** -0.5)
        with np.errstate(invalid="ignore"):
            ds = U * ((D + 12) * big + 8 * np.where(np.isfinite(rl), np.abs(rl), 0) + 8)
        steps = (len(s) + 64) * U
        tol = A * (B + 2 * ds[:, None] + steps) + B * np.abs(ref)
        assert np.all(np.abs(got[b] - ref) <= tol), (b, m, float(np.nanmax(np.abs(got[b] - ref) - tol)))
        if want_lse:
            fin = np.isfinite(rl)
            assert np.array_equal(gl[b][~fin], rl[~fin])
            assert np.all(np.abs(gl[b][fin] - rl[fin]) <= (ds + steps)[fin] + 4 * U * np.abs(rl[fin]))
    return O, lse, dev, attn


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("page", (16, 32, 64, 256))
def test_decode_lengths(mf, page, D, held):
    log(f"decode, pages of {page}, heads of {D}, {held}")
    lens = [0, 1, 2, 15, 16, 17, 31, 33, 100, 127, 128, 129, 0, 255, 256, 300, 700]
    check_decode(mf, Pages(mf, lens, 2, D, page, held, seed=page + D), lens, 6)


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("heads", [(1, 1), (5, 5), (8, 1), (16, 1), (17, 1), (40, 2), (128, 4), (256, 256)],
                         ids=str)
def test_decode_heads(mf, heads, held):
    log(f"decode, heads {heads}, {held}")
    lens = [200, 3, 0, 431]
    check_decode(mf, Pages(mf, lens, heads[1], 128, 64, held), lens, heads[0])


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("window", (1, 5, 16, 17, 100, 128, 5000))
def test_decode_windows(mf, window, held):
    log(f"decode, window {window}, {held}")
    lens = [0, 1, 50, 129, 1000, 333]
    check_decode(mf, Pages(mf, lens, 2, 64, 32, held), lens, 4, window)


@pytest.mark.parametrize("held", ("bf16", "mx8"))
def test_decode_long_and_many(mf, held):
    """Sequences that many workgroups share, and more sequences than threads."""
    log(f"decode, long, {held}")
    lens = [20000, 1, 3777]
    check_decode(mf, Pages(mf, lens, 2, 128, 128, held), lens, 8)
    lens = [(i * 37) % 150 for i in range(600)]
    log(f"decode, many, {held}")
    check_decode(mf, Pages(mf, lens, 1, 64, 16, held), lens, 2)


@pytest.mark.parametrize("held", ("bf16", "mx8"))
def test_decode_stale_pages_and_bad_entries(mf, held):
    """Pages full of NaN past the sequences' tokens, entries that stand for no page, tokens
    past the table's width."""
    t = torch()
    lens = [1, 17, 30, 200]
    p = Pages(mf, lens, 2, 64, 32, held, fill=float("nan"))
    x = t.randn(sum(lens), 4, 64, generator=gen(8)).to(t.bfloat16).cuda()
    mf.memfine_kv_write(p.cache, p.dtable, ints(lens), x[:, :2], x[:, 2:], offsets=ints(offsets_of(lens)))
    log(f"stale pages, {held}")
    O, lse, _, _ = check_decode(mf, p, lens, 4)
    assert t.all(t.isfinite(O.float()))
    p.table[3, 1], p.table[3, 4], p.table[1, 0] = -5, p.pages, 2 ** 31 - 1
    p.dtable = ints(p.table)
    log(f"entries that are no page, {held}")
    O, lse, _, _ = check_decode(mf, p, lens, 4)
    assert t.all(O[1] == 0) and t.all(lse[1] == -float("inf"))
    log(f"lengths outside, {held}")
    p = Pages(mf, [64, 64], 2, 64, 32, held)
    check_decode(mf, p, [-3, 10 ** 9], 4)


def test_decode_values_that_are_not_finite(mf):
    """A NaN key or value reaches its own sequence alone."""
    t = torch()
    lens = [300, 200, 500]
    p = Pages(mf, lens, 2, 64, 16, "bf16")
    O, lse, q, attn = check_decode(mf, p, lens, 4)
    for i in range(2):
        p.dev[i][p.table[1, 3]] = float("nan")
        P = t.zeros_like(O)
        log("a page of NaN")
        mf.memfine_attn_decode(attn, p.cache, p.dtable, ints(lens), q[:, :4], P)
        assert t.equal(P[[0, 2]], O[[0, 2]]) and t.all(t.isnan(P[1]))


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("D", (64, 128))
def test_decode_rounds_its_outputs_alone(mf, D, held):
    """The weights enter as two bf16 values, 2^-16 of each off: all that is left of bf16's half
    step is that of the output, also where a row's values cancel."""
    t = torch()
    lens, H = [7, 60, 300, 1500], 20
    p = Pages(mf, lens, 2, D, 32, held, seed=D)
    q = (t.randn(4, H, D, generator=gen(9)) * 1.5).to(t.bfloat16)
    O = t.full((4, H, D), float("nan"), dtype=t.bfloat16, device="cuda")
    log(f"weights of decode, {D} {held}")
    mf.memfine_attn_decode(mf.make_attn(H, 2, D), p.cache, p.dtable, ints(lens), q.cuda(), O)
    for b, n in enumerate(lens):
        ref, rl, A, big = at.decode(f64(q)[b], p.tokens(0, b, n), p.tokens(1, b, n), D ** -0.5)
        ds = U * ((D + 12) * big + 8 * np.abs(rl) + 8)
        tol = A * (2.0 ** -16 + 2 * ds[:, None] + (n + 64) * U) + B * np.abs(ref)
        off = np.abs(f64(O)[b] - ref) - tol
        assert np.all(off <= 0), (n, float(off.max()), int((off > 0).sum()))


def test_decode_is_the_same_causal_or_not(mf):
    t = torch()
    lens = [300, 0, 77]
    p = Pages(mf, lens, 2, 64, 32, "bf16")
    O, lse, q, _ = check_decode(mf, p, lens, 4)
    P, m = t.zeros_like(O), t.zeros_like(lse)
    log("not causal")
    mf.memfine_attn_decode(mf.make_attn(4, 2, 64, causal=False), p.cache, p.dtable, ints(lens), q[:, :4], P, m)
    assert t.equal(P, O) and t.equal(m, lse)
    with pytest.raises(mf.MemfineError):
        mf.memfine_attn_decode(mf.make_attn(4, 2, 64, causal=False, window=5), p.cache, p.dtable, ints(lens),
                               q[:, :4], P, m)


def test_decode_growing_scores(mf):
    t = torch()
    lens = [900]
    p = Pages(mf, lens, 1, 64, 64, "bf16")
    q = t.full((1, 3, 64), 1.0, dtype=t.bfloat16)
    for n in range(900):
        p.dev[0][p.table[0, n // 64], :, n % 64] = (n - 400) / 40
    log("growing scores")
    check_decode(mf, p, lens, 2, q=q)


def test_decode_again_streams_graphs_and_allocator(mf):
    t = torch()
    lens = [4000, 1, 0, 77, 1300]
    p = Pages(mf, lens, 4, 128, 64, "mx8")
    O, lse, q, attn = check_decode(mf, p, lens, 16)
    n = ints(lens)

    def call(out, l, **kw):
        mf.memfine_attn_decode(attn, p.cache, p.dtable, n, q[:, :16], out, l, **kw)
    side = t.cuda.Stream()
    P, m = t.zeros_like(O), t.zeros_like(lse)
    t.cuda.synchronize()
    log("side stream")
    with t.cuda.stream(side):
        call(P, m)
    side.synchronize()
    assert t.equal(P, O) and t.equal(m, lse)
    a = mf.TorchAllocator()
    call(P, m, allocator=a)
    assert t.equal(P, O) and not a.live
    assert a.high_water == mf.memfine_attn_decode_workspace_bytes(attn, p.cache, 5, p.width)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        call(P, m)
    more = [9000, 500]
    other = Pages(mf, more, 4, 128, 64, "bf16")
    for i in range(3):
        log(f"replay {i}")
        P.zero_()
        m.zero_()
        graph.replay()
        check_decode(mf, other, more, 8)
        assert t.equal(P, O) and t.equal(m, lse)
    # the graph follows the lengths
    n.copy_(ints([1, 1, 1, 1, 1]))
    graph.replay()
    check = [1] * 5
    O2, l2, _, _ = check_decode(mf, p, check, 16, q=q.cpu())
    assert t.equal(P, O2) and t.equal(m, l2)


def test_served_together(mf):
    """A prompt, then tokens one by one through the cache: each step's output is the
    last row of the attention over all rows so far."""
    t = torch()
    H, Hk, D, lens, steps = 8, 2, 128, [37, 5, 64], 4
    for held in ("bf16", "mx8"):
        p = Pages(mf, [n + steps for n in lens], Hk, D, 16, held)
        g = gen(12)
        cos, sin = (y.cuda() for y in tables(200, D))
        seqs = [t.randn(n + steps, H + 2 * Hk, D, generator=g).to(t.bfloat16).cuda() for n in lens]
        x = t.cat([s[:n] for s, n in zip(seqs, lens)])
        off = ints(offsets_of(lens))
        R = t.empty(len(x), H, D, dtype=t.bfloat16, device="cuda")
        mf.memfine_kv_write(p.cache, p.dtable, ints(lens), x[:, H:H + Hk], x[:, H + Hk:], offsets=off,
                            Q=x[:, :H], R=R, cos=cos, sin=sin)
        mf.memfine_rope(off, cos, sin, x[:, :H + Hk], x[:, :H + Hk])
        assert t.equal(R, x[:, :H])
        for i in range(steps):
            log(f"step {i} {held}")
            now = [n + i + 1 for n in lens]
            rows = t.stack([s[n - 1] for s, n in zip(seqs, now)])
            q = t.empty(len(lens), H, D, dtype=t.bfloat16, device="cuda")
            mf.memfine_kv_write(p.cache, p.dtable, ints(now), rows[:, H:H + Hk], rows[:, H + Hk:],
                                Q=rows[:, :H], R=q, cos=cos, sin=sin)
            O, _, _, _ = check_decode(mf, p, now, H, q=q.cpu())
        if held == "bf16":
            # over the rows themselves
            full = t.cat([s[:n + steps] for s, n in zip(seqs, lens)])
            off = ints(offsets_of([n + steps for n in lens]))
            mf.memfine_rope(off, cos, sin, full[:, :H + Hk], full[:, :H + Hk])
            P = t.empty(len(full), H, D, dtype=t.bfloat16, device="cuda")
            mf.memfine_attn_fwd(mf.make_attn(H, Hk, D), off, full[:, :H], full[:, H:H + Hk],
                                full[:, H + Hk:], P)
            last = (off[1:] - 1).long()
            # two roundings of the weights and of the output: 4 half steps of about 1
            assert t.allclose(P[last].float(), O.float(), rtol=2 ** -6, atol=2 ** -6)
