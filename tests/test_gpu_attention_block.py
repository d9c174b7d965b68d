"""The attention's calls together, as examples/moe_block.py runs them: served through the
cache (also from a captured graph) and trained, against torch in float64 on the same
weights."""
import os
import sys

import pytest

from gpu_harness import log, torch

pytestmark = pytest.mark.gpu
H, HK, D, HID = 8, 2, 64, 256


@pytest.fixture(scope="module")
def ex():
    t = torch()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import moe_block
    return moe_block


def draw(*shape, seed, std=1.0):
    t = torch()
    return (t.randn(*shape, generator=t.Generator().manual_seed(seed)) * std).to(t.bfloat16).cuda()


def turned(x, cos, sin, first=0):
    """Rows [n, heads, D] of one sequence in float64."""
    t = torch()
    c, s = (y[first:first + len(x)].double()[:, None] for y in (cos, sin))
    a, b = x[..., :D // 2], x[..., D // 2:]
    return t.cat([a * c - b * s, b * c + a * s], -1)


def attention64(qkv, cos, sin):
    """One sequence's rows [n, H + 2 HK, D] in float64, causal."""
    t = torch()
    qk = turned(qkv[:, :H + HK], cos, sin)
    q = qk[:, :H].transpose(0, 1)
    k, v = (y.transpose(0, 1).repeat_interleave(H // HK, 0) for y in (qk[:, H:], qkv[:, H + HK:]))
    s = t.matmul(q, k.transpose(1, 2).contiguous()) * D ** -0.5
    s = s.masked_fill(t.ones(s.shape[1:], dtype=t.bool, device=s.device).triu(1), -t.inf)
    return t.matmul(t.softmax(s, 2), v).transpose(0, 1).reshape(len(qkv), -1)


@pytest.mark.parametrize("mx8", (False, True), ids=("bf16", "mx8"))
def test_served_prompt_and_steps(ex, mx8):
    """Relative 2-norms: bf16 rounds qkv, the turned rows, weights and output by at most 2^-8
    each, 2^-6 in all; MX8 rounds keys and values by at most 2^-4 of each, by 2^-5
    on average over its steps, and what a score is off by enters all weights: 0.15."""
    t = torch()
    lens, steps = [37, 5, 100], 3
    W = draw((H + 2 * HK) * D, HID, seed=1, std=HID ** -0.5)
    a = ex.ServedAttention(W, ex.mf.make_attn(H, HK, D), 3, 128, page=32, mx8=mx8)
    held = t.empty(1, *W.shape, device="cuda")
    ex.mf.memfine_mxw_unpack(*a.W, held)
    W64 = held[0].double()
    rows = [draw(n + steps, HID, seed=10 + i) for i, n in enumerate(lens)]
    want = [attention64((r.double() @ W64.t()).view(len(r), -1, D), a.cos, a.sin) for r in rows]

    def off(got, ref):
        return ((got.double() - ref).norm() / ref.norm()).item()
    out = a.prompt(t.cat([r[:n] for r, n in zip(rows, lens)]), lens)
    log(f"prompts, mx8={mx8}")
    assert off(out, t.cat([w[:n] for w, n in zip(want, lens)])) <= 2 ** -6
    eager = []
    for i in range(steps):
        x = t.stack([r[n + i] for r, n in zip(rows, lens)])
        out = a.step(x)
        log(f"step {i}")
        assert off(out, t.stack([w[n + i] for w, n in zip(want, lens)])) <= (0.15 if mx8 else 2 ** -6)
        eager.append((x, out.clone()))
    # the same steps again, from a graph
    x = t.empty_like(eager[0][0])
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        a.step(x)
    a.lengths.copy_(t.tensor(lens))
    for i, (xi, o) in enumerate(eager):
        x.copy_(xi)
        graph.replay()
        t.cuda.synchronize()
        log(f"replay {i}")
        assert t.equal(a.out, o)


@pytest.mark.parametrize("mx8", (False, True), ids=("bf16", "mx8"))
def test_prompts_and_steps_cache_the_same_keys(ex, mx8):
    """A prompt's keys and values lie in the cache bit for bit as rows that are written with the
    tables in hand, as single tokens are: turned and rounded once."""
    t = torch()
    lens = [37, 5, 100]
    W = draw((H + 2 * HK) * D, HID, seed=1, std=HID ** -0.5)
    a, b = (ex.ServedAttention(W, ex.mf.make_attn(H, HK, D), 3, 128, page=32, mx8=mx8) for _ in range(2))
    x = draw(sum(lens), HID, seed=5)
    a.prompt(x, lens)
    qkv = t.empty(len(x), a.N, dtype=t.bfloat16, device="cuda")
    ex.mf.memfine_linear_mxw(a.N, a.h, x, *a.W, qkv)
    _, k, v = b.split(qkv)
    at = 0
    for i, n in enumerate(lens):      # token by token
        log(f"sequence {i}")
        for j in range(n):
            length = t.full((1,), j + 1, dtype=t.int32, device="cuda")
            ex.mf.memfine_kv_write(b.cache, b.table[i:i + 1], length, k[at + j:at + j + 1], v[at + j:at + j + 1],
                                   cos=b.cos, sin=b.sin)
        at += n
    for y, z in zip(a.cache.tensors, b.cache.tensors):
        assert (y is None and z is None) or t.equal(y, z)


def test_trained_gradients(ex):
    """Against autograd in float64: qkv, turned rows, attention's weights and outputs, the
    products' outputs are rounded to bf16, 2^-8 each at most: eight of them, 2^-5 of
    the 2-norm."""
    t = torch()
    lens = [50, 1, 77]
    T = sum(lens)
    Wqkv, Wo = draw((H + 2 * HK) * D, HID, seed=1, std=HID ** -0.5), draw(HID, H * D, seed=2, std=(H * D) ** -0.5)
    a = ex.TrainedAttention(Wqkv, Wo, ex.mf.make_attn(H, HK, D), lens)
    X, dout = draw(T, HID, seed=3), draw(T, HID, seed=4)
    out = a.forward(X)
    dX = a.backward(X, dout)
    x, w, o = (y.double().requires_grad_() for y in (X, Wqkv, Wo))
    qkv = (x @ w.t()).view(T, -1, D)
    ref = t.cat([attention64(q, a.cos, a.sin) for q in qkv.split(lens)]) @ o.t()
    grads = t.autograd.grad((ref * dout.double()).sum(), (x, w, o))
    log("trained")
    for name, got, want in (("out", out, ref), ("dX", dX, grads[0]), ("dWqkv", a.grads["Wqkv"], grads[1]),
                            ("dWo", a.grads["Wo"], grads[2])):
        rel = ((got.double() - want).norm() / want.norm()).item()
        assert rel <= 2 ** -5, (name, rel)


def test_layer_joins_attention_and_block(ex):
    """Served: the same bits as its calls one after the other.  Trained: the block's gradient goes
    through the attention and past it (a block that passes its input on, so that
    autograd in float64 knows the rest; tolerance as above)."""
    t = torch()
    gen = t.Generator(device="cuda").manual_seed(4)
    attn, tokens, E = ex.mf.make_attn(H, HK, D), 6, 16
    p = ex.weights(gen, HID, 128, E, H * D)
    gating = ex.mf.make_gating(E, 4, score="sigmoid", groups=4, top_groups=2, scale=2.5)
    W = ex.qkv_weight(gen, attn, HID)
    parts = [(ex.ServedAttention(W, attn, tokens, 64), ex.ServedBlock(**p, gating=gating, tokens=tokens))
             for _ in range(2)]
    w = draw(HID, seed=6)
    layer, (a, b) = ex.ServedLayer(w, *parts[0]), parts[1]
    x = draw(tokens * 20, HID, seed=7)
    a.prompt(x, [20] * tokens)
    layer.attention.prompt(x, [20] * tokens)
    stream, added = draw(tokens, HID, seed=8), draw(tokens, HID, seed=9)
    s2, a2 = stream.clone(), added.clone()
    for i in range(3):
        log(f"served layer, step {i}")
        added = layer.step(added, stream)
        y = t.empty_like(s2)
        ex.mf.memfine_norm_fwd(ex.EPS, a2, w, R=s2, S=s2, Y=y)
        a2 = b.step(a.step(y), s2)
        assert t.equal(added, a2) and t.equal(stream, s2) and bool(t.isfinite(added.float()).all())

    class Through:
        grads = {}

        def forward(self, X):
            return X

        def backward(self, X, dout):
            return dout
    lens = [30, 1, 40]
    Wo = draw(HID, H * D, seed=2, std=(H * D) ** -0.5)
    layer = ex.TrainedLayer(ex.TrainedAttention(W, Wo, attn, lens), Through())
    X, dout = draw(sum(lens), HID, seed=3), draw(sum(lens), HID, seed=4)
    log("trained layer")
    out = layer.forward(X)
    dX = layer.backward(X, dout)
    x, w, o = (y.double().requires_grad_() for y in (X, W, Wo))
    qkv = (x @ w.t()).view(len(X), -1, D)
    att = layer.attention
    ref = x + t.cat([attention64(q, att.cos, att.sin) for q in qkv.split(lens)]) @ o.t()
    grads = t.autograd.grad((ref * dout.double()).sum(), (x, w, o))
    for name, got, want in (("out", out, ref), ("dX", dX, grads[0]), ("dWqkv", layer.grads["Wqkv"], grads[1]),
                            ("dWo", layer.grads["Wo"], grads[2])):
        rel = ((got.double() - want).norm() / want.norm()).item()
        assert rel <= 2 ** -5, (name, rel)


def test_training_with_attention_moves_the_weights(ex):
    t = torch()
    gen = t.Generator(device="cuda").manual_seed(5)
    attn, E = ex.mf.make_attn(H, HK, D), 16
    p = ex.weights(gen, HID, 128, E, H * D)
    before = {n: v.clone() for n, v in p.items()}
    gating = ex.mf.make_gating(E, 4, score="sigmoid", groups=4, top_groups=2, scale=2.5)
    log("training with attention")
    losses = ex.train(p, gating, 101, 3, gen, lr=0.1, attn=attn)
    assert len(losses) == 3 and all(0 < x < float("inf") for x in losses)
    assert not any(t.equal(p[n], before[n]) for n in ("Wo", "Wr", "W1", "W2"))


def test_example_runs(ex, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["moe_block.py", "--tokens", "4", "--steps", "2", "--hidden", "256", "--ffn",
                                      "128", "--experts", "8", "--topk", "2", "--context", "40", "--heads", "4",
                                      "--kv-heads", "2"])
    ex.main()
    assert "attention: 4 sequences of 40 tokens" in capsys.readouterr().out
