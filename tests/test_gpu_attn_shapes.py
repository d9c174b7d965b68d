"""The attention's kernel shapes at the sizes that they are chosen for: workgroups of
eight waves and of many blocks, decode runs of more than 32 steps, and more sequences
than a wave plans by itself with several key-value heads and tiles of heads.

Tolerances are those of tests/test_gpu_attn.py and tests/test_gpu_cache.py."""
import numpy as np
import pytest

from gpu_harness import log, torch
from oracle import around as oa
from oracle import attention as at
from test_gpu_attn import FLUSHED, U, Case, f64, half_step, mf  # noqa: F401
from test_gpu_cache import B, Pages, check_decode, gen, ints

pytestmark = pytest.mark.gpu


def check_groups(c, groups):
    """Case.check for some key-value heads and the heads that share them."""
    share = c.H // c.Hk
    hs = [y * share + i for y in groups for i in range(share)]
    ys = list(groups)
    O, lse = c.forward()
    got = c.split(c.backward(O, lse))
    q, k, v = c.split(c.x)
    q, k, v, do = f64(q[:, hs]), f64(k[:, ys]), f64(v[:, ys]), f64(c.do[:, hs])
    o, ls = f64(O[:, hs]), f64(lse[hs])
    ref, rl, A, big = at.attn_fwd(q, k, v, c.off, c.scale, c.causal, c.window)
    r, n, b = c.rows, max(c.lens), half_step(c.dtype)
    ds = U * ((c.D + 12) * big + 8 * np.abs(rl) + 8)
    tol = A * ((b if c.dtype == "bf16" else 0.0) + 2 * ds.T[..., None] + (n + 8) * U) + b * np.abs(ref)
    off = np.abs(o[r] - ref[r]) - tol[r]
    assert np.all(off <= 0), float(np.nanmax(off))
    assert np.all((np.abs(ls - rl) - (ds + (n + 8) * U + 4 * U * np.abs(rl)))[:, r] <= 0)
    want, err = at.attn_bwd(q, k, v, np.where(r[:, None, None], o, 0), ls, do, c.off, c.scale, c.causal,
                            c.window, b if c.dtype == "bf16" else 0.0, U)
    for name, g, w, e, i in zip(("dQ", "dK", "dV"), got, want, err, (hs, ys, ys)):
        off = np.abs(f64(g[:, i])[r] - w[r]) - (e + b * np.abs(w))[r] - FLUSHED
        assert np.all(off <= 0), (name, float(np.nanmax(off)))
    for x in (O, *got):     # the other heads, and rows of no sequence
        assert bool(torch().isfinite(x[c.off[0]:c.off[-1]].float()).all())
        assert bool(torch().isnan(x[:c.off[0]]).all()) and bool(torch().isnan(x[c.off[-1]:]).all())


# (more than 1024 sets of 32 queries, so that no keys are shared out; heads of 64 with 2048
# rows a sequence or more go to workgroups of eight waves)
@pytest.mark.parametrize("kind", ("causal", "window", "all"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("lens,heads,groups", [([2100], (17, 17), (0, 16)), ([2305], (24, 8), (1, 7)),
                                               ([2500, 1700], (16, 2), (1,))], ids=str)
def test_long_sequences(mf, lens, heads, groups, D, kind):  # noqa: F811
    log(f"long {lens} {heads} {D} {kind}")
    kw = dict(causal=kind != "all", window=300 if kind == "window" else 0)
    check_groups(Case(mf, lens, *heads, D, "bf16", before=3, after=2, **kw), groups)


@pytest.mark.parametrize("kind", ("window", "all", "causal"))
@pytest.mark.parametrize("heads,groups", [((8, 2), (1,)), ((16, 4), (0, 3))], ids=str)
def test_few_heads_around_the_rule(mf, heads, groups, kind):  # noqa: F811
    """Two and four sets of 32 queries a compute unit: the keys are shared out among four
    waves, or not, as mask and window say."""
    log(f"few heads {heads} {kind}")
    kw = dict(causal=kind != "all", window=512 if kind == "window" else 0)
    check_groups(Case(mf, [2048], *heads, 128, "bf16", **kw), groups)


@pytest.mark.parametrize("D", (64, 128))
def test_long_sequences_fp32(mf, D):  # noqa: F811
    log(f"long fp32 {D}")
    check_groups(Case(mf, [1500, 3, 700], 6, 2, D, "f32"), (1,))


@pytest.mark.parametrize("held,D,window", [("mx8", 64, 0), ("bf16", 128, 0), ("mx8", 128, 39000)])
def test_decode_runs_of_many_steps(mf, held, D, window):  # noqa: F811
    """40000 tokens of 64 key-value heads: each workgroup goes through about 39 steps of 128, of
    whose pages it holds 32 steps' at a time."""
    t = torch()
    n, Hk, H, page = 40000, 64, 128, 64
    pages = n // page + 3
    size, g = (pages, Hk, page, D), t.Generator(device="cuda").manual_seed(D)
    sc = [None, None]
    if held == "bf16":
        kv = [t.randn(size, generator=g, device="cuda", dtype=t.bfloat16) for _ in range(2)]
    else:
        kv = [t.randint(0, 0x77, size, generator=g, device="cuda", dtype=t.uint8)
              | (t.randint(0, 2, size, generator=g, device="cuda", dtype=t.uint8) << 7) for _ in range(2)]
        sc = [t.randint(118, 122, (*size[:3], D // 32), generator=g, device="cuda", dtype=t.uint8)
              for _ in range(2)]
    cache = mf.make_cache(*kv, *sc)
    table = np.random.default_rng(1).permutation(pages)[None, :n // page]
    q = (t.randn(1, H, D, generator=gen(2)) * 1.5).to(t.bfloat16)
    O = t.full((1, H, D), float("nan"), dtype=t.bfloat16, device="cuda")
    lse = t.full((1, H), float("nan"), device="cuda")
    log(f"{n} tokens, {held}, heads of {D}, window {window}")
    mf.memfine_attn_decode(mf.make_attn(H, Hk, D, window=window), cache, ints(table), ints([n]), q.cuda(), O, lse)
    ids = t.from_numpy(table[0]).cuda()
    codes = np.concatenate([oa.e4m3_values(), [np.nan]])

    def values(i, y):
        x = kv[i][ids, y].cpu()
        if held == "bf16":
            return f64(x).reshape(-1, 1, D)
        x, s = x.numpy(), sc[i][ids, y].cpu().numpy().astype(np.float64)
        x = codes[x & 0x7f] * np.where(x & 0x80, -1, 1) * (2.0 ** (s - 127)).repeat(32, -1)
        return x.reshape(-1, 1, D)
    lo = max(0, n - window) if window else 0
    for y in (0, 1, 30, 63):
        hs = [2 * y, 2 * y + 1]
        ref, rl, A, big = at.decode(f64(q)[0, hs], values(0, y)[lo:], values(1, y)[lo:], D ** -0.5)
        ds = U * ((D + 12) * big + 8 * np.abs(rl) + 8)
        steps = (n + 64) * U
        tol = A * (B + 2 * ds[:, None] + steps) + B * np.abs(ref)
        assert np.all(np.abs(f64(O)[0, hs] - ref) <= tol), y
        assert np.all(np.abs(f64(lse)[0, hs] - rl) <= ds + steps + 4 * U * np.abs(rl)), y
    assert bool(t.isfinite(O.float()).all()) and bool(t.isfinite(lse).all())


@pytest.mark.parametrize("held", ("bf16", "mx8"))
@pytest.mark.parametrize("heads", [(40, 2), (6, 3), (51, 3)], ids=str)
@pytest.mark.parametrize("count", (64, 65, 100, 300))
def test_decode_of_many_sequences(mf, count, heads, held):  # noqa: F811
    """Sequences planned by a wave (64) and by a workgroup (more), with several key-value heads
    and, for groups of 17 and more, several tiles of heads; some sequences lie in several
    workgroups' runs, others are empty."""
    lens = [(i * 37) % 150 for i in range(count)]
    lens[3], lens[count // 2], lens[-1], lens[-2] = 2500, 1900, 700, 0
    log(f"decode, {count} sequences, heads {heads}, {held}")
    check_decode(mf, Pages(mf, lens, heads[1], 64, 32, held, seed=count), lens, heads[0])
