"""GPU parity of the attention over packed sequences against oracle/attention.py,
which starts from the same stored inputs in float64.

Tolerances, from the arithmetic (u = 2^-24, the fp32 unit; b the types' half step:
2^-8 for bf16, u for fp32):
* a score is a sum of dim products: off by (dim + 4) u of the sum of their magnitudes, B =
  max_j scale sum |q| |k|; a weight by that, by 4 u (|s| + |lse|) for the exponent's
  products, by 8 u for the power: ds = u ((dim + 4) B + 8 B + 8 |lse| + 8), twice (it
  enters the weights and their sum).
* O: the weights' rounding b (bf16 alone) and the errors above, with n + 8 steps of
  the sums, of sum_j p |v|, and b |O|: the output's rounding.
* lse: ds + (n + 8) u + 4 u |lse|.
* gradients: oracle.attention.attn_bwd's bounds, from the same units, and b of the
  value for the output's rounding.
* weights below the smallest normal float count as zero: 2^-126 each, times at most 2^13
  (|dp| + |delta|, scale < 1), 2^6 (|q|) and 2^9 terms: FLUSHED = 2^-98 of a gradient.
"""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import attention as oa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FLUSHED = 2.0 ** -98


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


def dtype_of(dtype):
    return torch().bfloat16 if dtype == "bf16" else torch().float32


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


class Case:
    """Packed rows whose queries, keys and values are columns of one tensor; `before`
    and `after` rows of no sequence."""

    def __init__(self, mf, lens, H, Hk, D, dtype, causal=True, window=0, seed=0, before=0, after=0,
                 q_std=1.5, k_std=1.0):
        t = torch()
        g = t.Generator().manual_seed(seed * 7919 + sum(lens) * 31 + H + D)
        self.lens, self.H, self.Hk, self.D, self.dtype = lens, H, Hk, D, dtype
        self.T = before + sum(lens) + after
        self.off = before + np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        x = t.randn(self.T, H + 2 * Hk, D, generator=g)
        x[:, :H] *= q_std
        x[:, H:H + Hk] *= k_std
        self.do = t.randn(self.T, H, D, generator=g).to(dtype_of(dtype))
        self.x = x.to(dtype_of(dtype))
        self.scale, self.causal, self.window = D ** -0.5, causal, window
        self.attn = mf.make_attn(H, Hk, D, causal=causal, window=window,
                                 dtype=mf.BF16 if dtype == "bf16" else mf.F32)
        self.mf = mf
        self.rows = np.zeros(self.T, bool)
        self.rows[self.off[0]:self.off[-1]] = True
        self.upload()

    def upload(self):
        t = torch()
        self.dev, self.ddo = self.x.cuda(), self.do.cuda()
        self.offsets = t.from_numpy(self.off).cuda()

    def split(self, x):
        return x[:, :self.H], x[:, self.H:self.H + self.Hk], x[:, self.H + self.Hk:]

    def forward(self, stream=None, fill=float("nan")):
        t = torch()
        O = t.full((self.T, self.H, self.D), fill, dtype=self.dev.dtype, device="cuda")
        lse = t.full((self.H, self.T), fill, device="cuda")
        self.mf.memfine_attn_fwd(self.attn, self.offsets, *self.split(self.dev), O, lse, stream=stream)
        return O, lse

    def backward(self, O, lse, fill=float("nan"), **kw):
        t = torch()
        d = t.full(self.dev.shape, fill, dtype=self.dev.dtype, device="cuda")
        self.mf.memfine_attn_bwd(self.attn, self.offsets, *self.split(self.dev), O, lse, self.ddo,
                                 *self.split(d), **kw)
        return d

    def check_forward(self, O, lse):
        q, k, v = (f64(x) for x in self.split(self.x))
        ref, rl, A, big = oa.attn_fwd(q, k, v, self.off, self.scale, self.causal, self.window)
        n = max(self.lens + [1])
        with np.errstate(invalid="ignore"):
            ds = U * ((self.D + 12) * big + 8 * np.abs(rl) + 8)
            lse_tol = ds + (n + 8) * U + 4 * U * np.abs(rl)
            b = half_step(self.dtype)
            tol = A * ((b if self.dtype == "bf16" else 0.0) + 2 * ds.T[..., None] + (n + 8) * U) + b * np.abs(ref)
        r = self.rows
        off = np.abs(f64(O)[r] - ref[r]) - tol[r]
        assert np.all(off <= 0), float(np.nanmax(off))
        assert np.all(np.abs(f64(lse)[:, r] - rl[:, r]) <= lse_tol[:, r])
        assert np.all(np.isnan(f64(O)[~r])) and np.all(np.isnan(f64(lse)[:, ~r]))

    def check_backward(self, O, lse, d):
        q, k, v = (f64(x) for x in self.split(self.x))
        b = half_step(self.dtype)
        want, err = oa.attn_bwd(q, k, v, np.where(self.rows[:, None, None], f64(O), 0), f64(lse),
                                f64(self.do), self.off, self.scale, self.causal, self.window,
                                b if self.dtype == "bf16" else 0.0, U)
        for name, got, w, e in zip(("dQ", "dK", "dV"), self.split(d), want, err):
            got = f64(got)
            off = np.abs(got[self.rows] - w[self.rows]) - (e + b * np.abs(w))[self.rows] - FLUSHED
            assert np.all(off <= 0), (name, float(np.nanmax(off)))
            assert np.all(np.isnan(got[~self.rows])), name

    def check(self):
        O, lse = self.forward()
        self.check_forward(O, lse)
        self.check_backward(O, lse, self.backward(O, lse))


LENS = [[1], [1, 1, 1], [2, 0, 31], [32, 33], [64], [65, 63, 1, 0, 0, 130], [255, 257], [300], [513]]


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths(mf, lens, D, dtype):
    log(f"lengths {lens} dim {D} {dtype}")
    Case(mf, lens, 2, 1, D, dtype).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (8, 8), (7, 1), (16, 2), (24, 8), (20, 5)], ids=str)
def test_heads(mf, heads, dtype):
    log(f"heads {heads} {dtype}")
    Case(mf, [70, 5, 129], *heads, 64 if heads[0] % 2 else 128, dtype).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("window", (1, 2, 31, 64, 100, 257, 2 ** 31 - 1))
def test_windows(mf, window, dtype):
    log(f"window {window} {dtype}")
    Case(mf, [300, 3, 0, 258], 4, 2, 128, dtype, window=window).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("D", (64, 128))
def test_not_causal(mf, D, dtype):
    log(f"not causal {D} {dtype}")
    Case(mf, [1, 95, 0, 300], 4, 2, D, dtype, causal=False).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_rows_of_no_sequence_are_left(mf, dtype):
    log(f"rows before and after {dtype}")
    Case(mf, [40, 0, 77], 4, 2, 128, dtype, before=5, after=70).check()


@pytest.mark.parametrize("count", (63, 64, 65, 700, 4200))
def test_many_sequences(mf, count):
    log(f"{count} sequences")
    lens = [(i * 7) % 4 for i in range(count)]
    Case(mf, lens, 2, 1, 64, "bf16").check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_large_scores_and_a_growing_maximum(mf, dtype):
    """Scores of hundreds, whose maximum rises from tile to tile: the sums move along."""
    log(f"large scores {dtype}")
    c = Case(mf, [400], 2, 1, 64, dtype, q_std=8.0, k_std=4.0)
    c.x[:, 2] *= t_ramp(400, c.x.dtype)
    c.upload()
    c.check()


def t_ramp(n, dtype):
    return torch().linspace(0.01, 1.5, n)[:, None].to(dtype)


def test_offsets_outside_are_cut(mf):
    """Offsets that do not ascend or leave [0, T]: nothing outside is touched, and
    what they hold of the rows is computed."""
    t = torch()
    c = Case(mf, [64, 64], 2, 1, 64, "bf16")
    O, lse = c.forward()
    c.offsets = t.tensor([-9, 64, 100000], dtype=t.int32, device="cuda")
    log("offsets outside")
    P, m = c.forward()
    assert t.equal(O, P) and t.equal(lse, m)
    c.offsets = t.tensor([128, 64, 0], dtype=t.int32, device="cuda")
    P, m = c.forward()
    assert t.all(t.isnan(P)) and t.all(t.isnan(m))


def test_a_sequence_that_is_not_finite_stays_alone(mf):
    t = torch()
    c = Case(mf, [100, 61, 90], 4, 2, 128, "bf16")
    O, lse = c.forward()
    d = c.backward(O, lse)
    for bad in (float("nan"), float("inf")):
        c.x[100:161] = bad
        c.do[100:161] = bad
        c.upload()
        log(f"a sequence of {bad}")
        P, m = c.forward()
        e = c.backward(P, m)
        keep = [i for i in range(251) if not 100 <= i < 161]
        assert t.equal(P[keep], O[keep]) and t.equal(m[:, keep], lse[:, keep])
        assert t.equal(e[keep], d[keep])
        assert not t.any(t.isfinite(P[100:161].float()))


def test_same_results_again_and_contiguous(mf):
    """Bit for bit: run again, and with contiguous operands."""
    t = torch()
    c = Case(mf, [500, 129, 1], 8, 2, 128, "bf16")
    O, lse = c.forward()
    d = c.backward(O, lse)
    log("again")
    P, m = c.forward()
    e = c.backward(P, m)
    assert t.equal(O, P) and t.equal(lse, m) and t.equal(d, e)
    q, k, v = (x.contiguous() for x in c.split(c.dev))
    mf.memfine_attn_fwd(c.attn, c.offsets, q, k, v, P)
    assert t.equal(O, P)
    out = [t.full_like(x, float("nan")) for x in (q, k, v)]
    mf.memfine_attn_bwd(c.attn, c.offsets, q, k, v, O, lse, c.ddo, *out)
    assert all(t.equal(a, b) for a, b in zip(out, c.split(d)))


def test_streams_graphs_and_allocator(mf):
    """On a side stream, from a captured graph whose replays follow other eager work,
    and with the caller's allocator."""
    t = torch()
    c = Case(mf, [333, 40], 8, 2, 64, "bf16")
    O, lse = c.forward()
    d = c.backward(O, lse)
    side = t.cuda.Stream()
    t.cuda.synchronize()
    log("side stream")
    with t.cuda.stream(side):
        P, m = c.forward()
        e = c.backward(P, m)
    side.synchronize()
    assert t.equal(O, P) and t.equal(lse, m) and t.equal(d, e)
    a = mf.TorchAllocator()
    e = c.backward(O, lse, allocator=a)
    assert t.equal(d, e) and not a.live
    assert a.high_water == mf.memfine_attn_bwd_workspace_bytes(c.attn, c.T, 2)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        P, m = c.forward()
        e = c.backward(P, m)
    other = Case(mf, [700], 8, 2, 64, "bf16", seed=3)
    for i in range(3):
        log(f"replay {i}")
        for x in (P, m, e):
            x.fill_(float("nan"))
        graph.replay()
        other.backward(*other.forward())
        t.cuda.synchronize()
        assert t.equal(O, P) and t.equal(lse, m) and t.equal(d, e)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_parts_of_the_queries(mf, dtype):
    """Few keys and many queries to them: these are shared out and the sums added."""
    log(f"parts, {dtype}")
    c = Case(mf, [700, 0, 433], 32, 1, 64, dtype, before=3, after=2)
    c.check()
    need = mf.memfine_attn_bwd_workspace_bytes
    parts = (need(c.attn, 1138, 3) - 2 * 1138 * 32 * 4) / (2 * 1138 * 64 * 4)
    assert parts == int(parts) and parts >= 2
    Case(mf, [1300], 14, 2, 128, dtype).check()        # seven heads, not a power of two
    Case(mf, [3, 1, 0, 40], 24, 1, 128, dtype).check()  # parts without a tile
    Case(mf, [900], 1, 1, 64, dtype).check()           # one head's queries in parts
    Case(mf, [1500, 130], 2, 2, 128, dtype, window=70).check()


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (8, 1)], ids=str)
@pytest.mark.parametrize("kind", ("causal", "window", "all"))
def test_few_queries(mf, heads, D, kind):
    """Few heads of long sequences, whose keys four waves share: lengths around the tiles,
    a short sequence beside them, rows of no sequence, large scores that grow."""
    t = torch()
    kw = dict(causal=kind != "all", window=200 if kind == "window" else 0)
    log(f"few queries, {heads} {D} {kind}")
    for lens in ([513], [1000, 7, 0, 897], [640, 385]):
        Case(mf, lens, *heads, D, "bf16", before=2, after=1, **kw).check()
    c = Case(mf, [800], *heads, D, "bf16", q_std=6.0, k_std=3.0, **kw)
    c.x[:, heads[0]] *= t_ramp(800, c.x.dtype)
    c.upload()
    c.check()
    O, lse = c.forward()
    P, m = c.forward()
    assert t.equal(O, P) and t.equal(lse, m)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (16, 4)], ids=str)
def test_one_visible_token_has_no_gradient_of_scores(mf, heads, D):
    """bf16: where a token sees itself alone its weight is 1 and its output the value, so
    that dp - delta, of equal rows summed in one order, is zero: dQ is exactly zero for a
    sequence's first token, and dQ and dK for a window of one and sequences of one."""
    t = torch()
    for lens, window in (([1] * 37, 0), ([300, 1, 64], 1), ([900], 1), ([900], 0), ([5, 70, 33], 0)):
        log(f"one visible token, {heads} {D} {lens[0]} x {len(lens)} window {window}")
        c = Case(mf, lens, *heads, D, "bf16", window=window, before=1)
        O, lse = c.forward()
        d = c.backward(O, lse)
        dQ, dK, _ = c.split(d)
        rows = t.from_numpy(c.rows).cuda()
        if max(lens) == 1 or window == 1:
            assert int(t.count_nonzero(dQ[rows])) == 0 and int(t.count_nonzero(dK[rows])) == 0
        else:
            assert int(t.count_nonzero(dQ[c.offsets[:-1].long()])) == 0
        c.check_backward(O, lse, d)


def test_gradient_against_differences(mf):
    """fp32: the loss sum(O dO) along random directions; a step of e leaves a second
    difference of e^2 and rounding of about 2^-24 sum |O dO| / e."""
    t = torch()
    c = Case(mf, [50, 17], 4, 2, 64, "f32")
    O, lse = c.forward()
    d = f64(c.backward(O, lse))
    x0, e = c.dev.clone(), 2.0 ** -7
    for seed in range(6):
        log(f"direction {seed}")
        r = t.randn(x0.shape, generator=t.Generator().manual_seed(seed)).cuda()
        part = (t.arange(x0.shape[1]) % 3 == seed % 3).cuda()[None, :, None]
        r = r * part
        ups = []
        for s in (1, -1, 2, -2):
            c.dev = x0 + s * e * r
            ups.append(float((f64(c.forward()[0]) * f64(c.do)).sum()))
        # fourth order: (8 (f(e) - f(-e)) - (f(2e) - f(-2e))) / 12 e
        num = (8 * (ups[0] - ups[1]) - (ups[2] - ups[3])) / (12 * e)
        want = float((d * f64(r)).sum())
        size = np.sqrt((d * d * f64(r) ** 2).sum())
        assert abs(num - want) <= 2e-2 * max(size, abs(want)), (num, want)
