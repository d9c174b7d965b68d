"""Attention in front of the expert layer, as measurable calls.

Three operators that a block needs between its projections and the experts:

* ``prompt``  attention over packed sequences of different lengths, causal or
              not, a window of the last tokens, key-value heads shared by
              groups of heads; forward and backward.
* ``decode``  attention of one new token a sequence over a cache of pages, held
              in bf16 or in MX8 (e4m3 values, one power-of-two scale per 32).
* ``rotary``  the rotation of queries and keys by their positions: rows of a
              packed batch, forward and backward ("rope"), or new tokens on
              their way into the cache ("write").

Every case is one call of one of them (and, for an MX8 cache that was written,
the call that gives its values).  With ``own`` unset `run` computes the operator
from elementary torch operations in float32; with it set it calls the library.
`exact` gives the same outputs from the definitions in float64.

Definitions, for a token i of a sequence of n (heads j of a group share a
key-value head; lse is the logarithm of the weights' sum):

    s_ij = scale q_i . k_j;  j <= i (causal);  j > i - window (where there is one)
    o_i = sum_j exp(s_ij - lse_i) v_j;   lse_i = log sum_j exp(s_ij)

A rotation turns the pairs (x_i, x_{i + dim/2}), or (x_{2i}, x_{2i+1}) where it is
interleaved, by the angle whose cosine and sine the tables hold for the position.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # Three short prompts in one batch, one of them a single token: latency.
        dict(name="prompt_short", op="prompt", back=False, T=101, seqs=3, heads=32, kv_heads=8,
             dim=128, causal=True, window=0, dtype="bf16"),
        # Twelve prompts of 90 to 2000 tokens, packed, an odd number of tokens in all.
        dict(name="prompt_packed", op="prompt", back=False, T=8191, seqs=12, heads=32, kv_heads=8,
             dim=128, causal=True, window=0, dtype="bf16"),
        # A whole sequence of 4096 with the 128 heads of 128 of the paper's Model I, in training.
        dict(name="prompt_heads128", op="prompt", back=False, T=4096, seqs=1, heads=128,
             kv_heads=128, dim=128, causal=True, window=0, dtype="bf16"),
        # Its gradient, heads in groups of eight.
        dict(name="prompt_backward", op="prompt", back=True, T=4096, seqs=1, heads=64, kv_heads=8,
             dim=128, causal=True, window=0, dtype="bf16"),
        # The gradient of packed sequences of uneven lengths, small heads, a window.
        dict(name="prompt_backward_ragged", op="prompt", back=True, T=6011, seqs=9, heads=16,
             kv_heads=16, dim=64, causal=True, window=512, dtype="bf16"),
        # One sequence's next token: latency.
        dict(name="decode_1", op="decode", seqs=1, total=2049, heads=32, kv_heads=8, dim=128,
             window=0, page=64, held="bf16"),
        # The same far into a document.
        dict(name="decode_long", op="decode", seqs=1, total=131072, heads=32, kv_heads=8, dim=128,
             window=0, page=256, held="bf16"),
        # A serving batch of very different lengths, small pages, the cache in MX8.
        dict(name="decode_batch", op="decode", seqs=64, total=262139, heads=64, kv_heads=8,
             dim=128, window=0, page=16, held="mx8"),
        # Sixteen sequences of the paper's Model I: no shared heads, the most cache a token.
        dict(name="decode_heads128", op="decode", seqs=16, total=32768, heads=128, kv_heads=128,
             dim=128, window=0, page=128, held="bf16"),
        # The new tokens of a decode batch, rotated, into the cache: latency.
        dict(name="write_decode", op="write", T=64, seqs=64, past=500, heads=32, kv_heads=8,
             dim=128, page=64, held="bf16", interleaved=False),
        # A prefill's rows, rotated, into an MX8 cache.
        dict(name="write_prefill", op="write", T=8191, seqs=5, past=0, heads=64, kv_heads=8,
             dim=128, page=64, held="mx8", interleaved=False),
        # Queries and keys of a training batch with the paper's heads, turned back (the gradient).
        dict(name="rope_backward", op="rope", T=8192, seqs=2, heads=256, dim=128, dtype="bf16",
             inverse=True, interleaved=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("prompt", "prompt", "prompt", "decode", "decode", "rotary"))
    dim = rng.choice((64, 128, 128))
    kv = rng.choice((1, 2, 4, 8, 8, 16))
    group = rng.choice((1, 1, 2, 4, 7, 8, 16))
    if op == "prompt":
        while True:
            T, back = _log_int(rng, 1, 8192), rng.random() < 0.45
            dtype = "f32" if rng.random() < 0.15 else "bf16"
            causal = rng.random() < 0.8
            c = dict(op=op, back=back, T=T, seqs=min(T, _log_int(rng, 1, 24)), heads=kv * group,
                     kv_heads=kv, dim=dim, causal=causal,
                     window=_log_int(rng, 16, 2048) if causal and rng.random() < 0.3 else 0,
                     dtype=dtype)
            # the plain form holds all pairs of a sequence
            most = max(_lengths(T, c["seqs"]))
            if (3 if back else 1) * (6 if dtype == "f32" else 1) * c["heads"] * T * most <= 2e9:
                return c
            kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 8))
    held = rng.choice(("bf16", "mx8"))
    page = rng.choice((16, 32, 64, 128, 256))
    if op == "decode":
        seqs = _log_int(rng, 1, 128)
        while True:
            total = max(seqs, _log_int(rng, 8, 400000))
            if total * kv * dim <= 2.7e8:
                break
        return dict(op=op, seqs=seqs, total=total, heads=kv * group, kv_heads=kv, dim=dim,
                    window=_log_int(rng, 16, 4096) if rng.random() < 0.25 else 0, page=page,
                    held=held)
    if rng.random() < 0.5:
        T = _log_int(rng, 1, 8192)
        return dict(op="rope", T=T, seqs=min(T, _log_int(rng, 1, 24)), heads=kv * (group + 1),
                    dim=dim, dtype="f32" if rng.random() < 0.3 else "bf16",
                    inverse=rng.random() < 0.5, interleaved=rng.random() < 0.5)
    T = _log_int(rng, 1, 8192)
    seqs = T if T <= 128 and rng.random() < 0.5 else min(T, _log_int(rng, 1, 24))
    return dict(op="write", T=T, seqs=seqs, past=_log_int(rng, 1, 1000) - 1, heads=kv * group,
                kv_heads=kv, dim=dim, page=page, held=held, interleaved=rng.random() < 0.5)


def _lengths(total, n):
    """n uneven lengths, one at least each, that add up to total."""
    w = [0.05 + ((i * 0.6180339887498949 + 0.9) % 1.0) ** 2 for i in range(n)]
    left = total - n
    out = [1 + int(left * x / sum(w)) for x in w]
    out[max(range(n), key=lambda i: w[i])] += total - sum(out)
    return out


# ----------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 71)
    return g


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n].copy_(torch.randn(n, generator=gen, device="cuda") * std)
    return x


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return _ints(at)


def _mx8_rows(x):
    """x [rows, h] as MX8: e4m3 bytes [rows, h] and scale bytes [rows, h/32], the
    scale the smallest power of two 2^e for which max|x| <= 448 * 2^e."""
    b = x.float().view(x.shape[0], -1, 32)
    m, ex = torch.frexp(b.abs().amax(2))
    e = (ex - 9 + (m > 0.875).int()).clamp(min=-127)
    q = torch.ldexp(b, -e[..., None]).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).view(x.shape), (e + 127).to(torch.uint8)


def _mx8_values(q, s):
    """float32 values of e4m3 bytes [..., h] with scale bytes [..., h/32]."""
    b = q.view(torch.float8_e4m3fn).float().view(*s.shape, 32)
    return torch.ldexp(b, s.int()[..., None] - 127).view(q.shape)


def _tables(positions, dim):
    """Cosines and sines [positions, dim / 2], from angles in float64."""
    f = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cos(a).float(), torch.sin(a).float()


def _paged(c, gen, lens):
    """A cache of the pages that sequences of these lengths need, in a shuffled
    order, full of normal values, and the sequences' table."""
    need = [-(-n // c["page"]) for n in lens]
    pages, width = sum(need) + 3, max(need) + 1
    order = torch.randperm(pages, generator=gen, device="cuda").tolist()
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-1] * (width - n))
        at += n
    s = {"table": _ints(rows)}
    size = (pages, c["kv_heads"], c["page"], c["dim"])
    for name in ("k", "v"):
        x = _normal(gen, size, 1.0, torch.bfloat16)
        if c["held"] == "bf16":
            s["c" + name], s["c" + name + "s"] = x, None
        else:
            q, e = _mx8_rows(x.view(-1, c["dim"]))
            s["c" + name], s["c" + name + "s"] = q.view(size), e.view(*size[:3], c["dim"] // 32)
    if own:
        import paper_2511_21431_amd as mf
        s["cache"] = mf.make_cache(s["ck"], s["cv"], s["cks"], s["cvs"])
    return s


def prepare(case, seed):
    c, gen, dev = case, _gen(seed), "cuda"
    s = dict(case)
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    D = c["dim"]
    if c["op"] == "prompt":
        T, H, Hk = c["T"], c["heads"], c["kv_heads"]
        s["lens"] = _lengths(T, c["seqs"])
        s["offsets"] = _offsets(s["lens"])
        # queries, keys and values side by side in a row, as one projection writes them
        qkv = _normal(gen, (T, H + 2 * Hk, D), 1.0, dt)
        qkv[:, :H] *= 1.5
        s["Q"], s["K"], s["V"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        s["scale"] = D ** -0.5
        s["O"] = torch.empty((T, H, D), dtype=dt, device=dev)
        s["lse"] = torch.empty((H, T), device=dev)
        if own:
            import paper_2511_21431_amd as mf
            s["attn"] = mf.make_attn(H, Hk, D, causal=c["causal"], window=c["window"],
                                     scale=s["scale"], dtype=mf.F32 if dt == torch.float32 else mf.BF16)
        if c["back"]:
            f = _prompt_plain(s)
            s["O"], s["lse"] = f["O"], f["lse"]
            s["dO"] = _normal(gen, (T, H, D), 1.0, dt)
            d = torch.empty((T, H + 2 * Hk, D), dtype=dt, device=dev)
            s["dQ"], s["dK"], s["dV"] = d[:, :H], d[:, H:H + Hk], d[:, H + Hk:]
        return s
    if c["op"] == "decode":
        lens = _lengths(c["total"], c["seqs"])
        s["lens"], s["lengths"] = lens, _ints(lens)
        s.update(_paged(c, gen, lens))
        s["scale"] = D ** -0.5
        s["Q"] = _normal(gen, (c["seqs"], c["heads"], D), 1.5, torch.bfloat16)
        s["O"] = torch.empty_like(s["Q"])
        if own:
            import paper_2511_21431_amd as mf
            s["attn"] = mf.make_attn(c["heads"], c["kv_heads"], D, causal=True, window=c["window"],
                                     scale=s["scale"])
        return s
    lens = _lengths(c["T"], c["seqs"])
    s["lens"], s["offsets"] = lens, _offsets(lens)
    if c["op"] == "rope":
        s["cos"], s["sin"] = _tables(max(lens), D)
        s["X"] = _normal(gen, (c["T"], c["heads"], D), 1.0, dt)
        s["Y"] = torch.empty_like(s["X"])
        return s
    H, Hk = c["heads"], c["kv_heads"]
    ends = [n + c["past"] for n in lens]
    s["lengths"] = _ints(ends)
    s["cos"], s["sin"] = _tables(max(ends), D)
    s.update(_paged(c, gen, ends))
    qkv = _normal(gen, (c["T"], H + 2 * Hk, D), 1.0, torch.bfloat16)
    s["Q"], s["K"], s["V"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    s["R"] = torch.empty((c["T"], H, D), dtype=torch.bfloat16, device=dev)
    if c["held"] == "mx8":
        s["kv"] = torch.empty((2, *s["ck"].shape), dtype=torch.bfloat16, device=dev)
    return s


# ------------------------------------------------------------- plain forms
def _hidden(c, n, dev):
    """[n, n], true where token i does not see token j."""
    i, j = torch.arange(n, device=dev)[:, None], torch.arange(n, device=dev)
    off = (j > i) if c["causal"] else torch.zeros((n, n), dtype=torch.bool, device=dev)
    return off | (j <= i - c["window"]) if c["window"] else off


def _sequences(s):
    """(rows, key-value heads) of the parts that the plain forms take at once."""
    at = 0
    for n in s["lens"]:
        step = max(1, int(2 ** 29 // (n * n * (s["heads"] // s["kv_heads"]))))
        for h in range(0, s["kv_heads"], step):
            yield slice(at, at + n), slice(h, min(h + step, s["kv_heads"]))
        at += n


def _grouped(s, x, rows, kv):
    """The heads of these key-value heads, float32 [kv heads, group * rows, dim]."""
    g = s["heads"] // s["kv_heads"]
    x = x[rows, kv.start * g:kv.stop * g].float()
    n = x.shape[0]
    return x.reshape(n, -1, g, s["dim"]).permute(1, 2, 0, 3).reshape(-1, g * n, s["dim"]).contiguous()


def _ungrouped(s, x, n):
    g = s["heads"] // s["kv_heads"]
    return x.view(-1, g, n, s["dim"]).permute(2, 0, 1, 3).reshape(n, -1, s["dim"])


def _weights(s, q, k, off):
    n = off.shape[0]
    z = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
    return z.view(z.shape[0], -1, n, n).masked_fill_(off, -torch.inf).view(z.shape)


def _prompt_plain(s):
    O, lse = torch.empty_like(s["O"]), torch.empty_like(s["lse"])
    g = s["heads"] // s["kv_heads"]
    for rows, kv in _sequences(s):
        n = rows.stop - rows.start
        q = _grouped(s, s["Q"], rows, kv)
        k, v = (s[x][rows, kv].float().transpose(0, 1).contiguous() for x in "KV")
        z = _weights(s, q, k, _hidden(s, n, q.device))
        m = z.amax(2, keepdim=True)
        p = torch.exp(z - m)
        t = p.sum(2, keepdim=True)
        heads = slice(kv.start * g, kv.stop * g)
        O[rows, heads] = _ungrouped(s, torch.matmul(p, v) / t, n).to(O.dtype)
        lse[heads, rows] = (m + torch.log(t)).view(-1, n)
    return {"O": O, "lse": lse}


def _prompt_back_plain(s):
    dQ, dK, dV = (torch.empty(s[x].shape, dtype=s[x].dtype, device=s[x].device) for x in "QKV")
    g = s["heads"] // s["kv_heads"]
    for rows, kv in _sequences(s):
        n = rows.stop - rows.start
        heads = slice(kv.start * g, kv.stop * g)
        q, o, do = (_grouped(s, s[x], rows, kv) for x in ("Q", "O", "dO"))
        k, v = (s[x][rows, kv].float().transpose(0, 1).contiguous() for x in "KV")
        p = torch.exp(_weights(s, q, k, _hidden(s, n, q.device))
                      - s["lse"][heads, rows].reshape(kv.stop - kv.start, g * n, 1))
        dV[rows, kv] = torch.matmul(p.transpose(1, 2).contiguous(), do).transpose(0, 1).to(dV.dtype)
        dz = torch.matmul(do, v.transpose(1, 2).contiguous())
        dz = p * (dz - (do * o).sum(2, keepdim=True)) * s["scale"]
        dQ[rows, heads] = _ungrouped(s, torch.matmul(dz, k), n).to(dQ.dtype)
        dK[rows, kv] = torch.matmul(dz.transpose(1, 2).contiguous(), q).transpose(0, 1).to(dK.dtype)
    return {"dQ": dQ, "dK": dK, "dV": dV}


def _cached(s, b, name, lo):
    """float32 [kv heads, tokens from lo on, dim] of sequence b."""
    n, page = s["lens"][b], s["page"]
    first = lo // page
    ids = s["table"][b, first:-(-n // page)].long()
    x, e = s["c" + name][ids], s["c" + name + "s"]
    x = x.float() if e is None else _mx8_values(x, e[ids])
    x = x.transpose(0, 1).reshape(s["kv_heads"], -1, s["dim"])
    return x[:, lo - first * page:n - first * page].contiguous()


def _decode_plain(s):
    O = torch.empty_like(s["O"])
    for b, n in enumerate(s["lens"]):
        lo = max(0, n - s["window"]) if s["window"] else 0
        q = s["Q"][b].float().view(s["kv_heads"], -1, s["dim"])
        z = torch.matmul(q, _cached(s, b, "k", lo).transpose(1, 2).contiguous()) * s["scale"]
        p = torch.exp(z - z.amax(2, keepdim=True))
        o = torch.matmul(p, _cached(s, b, "v", lo)) / p.sum(2, keepdim=True)
        O[b] = o.view(-1, s["dim"]).to(O.dtype)
    return {"O": O}


def _turn(x, cos, sin, interleaved):
    """Rows x [rows, heads, dim] with the rows' cosines and sines [rows, dim / 2]."""
    x, c, n = x.float(), cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * c - b * n, b * c + a * n), -1)


def _positions(s, past=0):
    return torch.cat([torch.arange(past, past + n, device="cuda") for n in s["lens"]])


def _rope_plain(s):
    at = _positions(s)
    sin = s["sin"][at]
    return {"Y": _turn(s["X"], s["cos"][at], -sin if s["inverse"] else sin,
                       s["interleaved"]).to(s["X"].dtype)}


def _write_plain(s):
    at = _positions(s, s["past"])
    cos, sin = s["cos"][at], s["sin"][at]
    seq = torch.repeat_interleave(torch.arange(s["seqs"], device="cuda"),
                                  torch.tensor(s["lens"], device="cuda"), output_size=s["T"])
    page, row = s["table"][seq, at // s["page"]].long(), at % s["page"]
    for name, x in (("k", _turn(s["K"], cos, sin, s["interleaved"])), ("v", s["V"].float())):
        if s["held"] == "bf16":
            s["c" + name][page, :, row] = x.to(torch.bfloat16)
        else:
            q, e = _mx8_rows(x.reshape(-1, s["dim"]))
            s["c" + name][page, :, row] = q.view(x.shape)
            s["c" + name + "s"][page, :, row] = e.view(*x.shape[:2], -1)
    out = {"Q": _turn(s["Q"], cos, sin, s["interleaved"]).to(torch.bfloat16)}
    for name in ("k", "v"):
        out[name] = s["c" + name] if s["held"] == "bf16" else \
            _mx8_values(s["c" + name], s["c" + name + "s"]).to(torch.bfloat16)
    return out


# --------------------------------------------------------------------- run
def run(state):
    s = state
    if not own:
        if s["op"] == "prompt":
            return _prompt_back_plain(s) if s["back"] else _prompt_plain(s)
        return {"decode": _decode_plain, "rope": _rope_plain, "write": _write_plain}[s["op"]](s)
    import paper_2511_21431_amd as mf
    if s["op"] == "prompt" and s["back"]:
        mf.memfine_attn_bwd(s["attn"], s["offsets"], s["Q"], s["K"], s["V"], s["O"], s["lse"],
                            s["dO"], s["dQ"], s["dK"], s["dV"])
        return {"dQ": s["dQ"], "dK": s["dK"], "dV": s["dV"]}
    if s["op"] == "prompt":
        mf.memfine_attn_fwd(s["attn"], s["offsets"], s["Q"], s["K"], s["V"], s["O"], s["lse"])
        return {"O": s["O"], "lse": s["lse"]}
    if s["op"] == "decode":
        mf.memfine_attn_decode(s["attn"], s["cache"], s["table"], s["lengths"], s["Q"], s["O"])
        return {"O": s["O"]}
    if s["op"] == "rope":
        mf.memfine_rope(s["offsets"], s["cos"], s["sin"], s["X"], s["Y"],
                        interleaved=s["interleaved"], inverse=s["inverse"])
        return {"Y": s["Y"]}
    # one row a sequence needs no offsets
    mf.memfine_kv_write(s["cache"], s["table"], s["lengths"], s["K"], s["V"],
                        offsets=None if s["T"] == s["seqs"] else s["offsets"], Q=s["Q"], R=s["R"],
                        cos=s["cos"], sin=s["sin"], interleaved=s["interleaved"])
    if s["held"] == "bf16":
        return {"Q": s["R"], "k": s["ck"], "v": s["cv"]}
    D = s["dim"]
    for i, name in enumerate(("k", "v")):
        mf.memfine_mx_values(s["c" + name].view(-1, D), s["c" + name + "s"].view(-1, D // 32),
                             s["kv"][i].view(-1, D))
    return {"Q": s["R"], "k": s["kv"][0], "v": s["kv"][1]}


def _seen(c, n):
    """Pairs (i, j) of a sequence of n, token i sees token j."""
    if not c["causal"]:
        return n * n
    w = min(n, c["window"] or n)
    return w * (w + 1) // 2 + (n - w) * w


def work(case):
    c = case
    D, H = c["dim"], c["heads"]
    if c["op"] == "prompt":
        Hk, es = c["kv_heads"], 4 if c["dtype"] == "f32" else 2
        pairs = sum(_seen(c, n) for n in _lengths(c["T"], c["seqs"]))
        rows = c["T"] * (H + Hk)  # queries and outputs, or keys and values
        if c["back"]:  # Q, K, V, O, dO and the gradients of the first three; lse
            return {"bytes": 2.0 * es * D * (rows + c["T"] * (H + Hk)) + 4.0 * c["T"] * H,
                    "flops": 10.0 * D * H * pairs}
        return {"bytes": 2.0 * es * D * rows + 4.0 * c["T"] * H, "flops": 4.0 * D * H * pairs}
    if c["op"] == "decode":
        n = sum(min(x, c["window"] or x) for x in _lengths(c["total"], c["seqs"]))
        per = 2 * D if c["held"] == "bf16" else D + D // 32
        return {"bytes": 2.0 * n * c["kv_heads"] * per + 4.0 * c["seqs"] * H * D,
                "flops": 4.0 * D * H * n}
    if c["op"] == "rope":
        n = c["T"] * H * D
        return {"bytes": 2.0 * n * (4 if c["dtype"] == "f32" else 2)
                + 4.0 * max(_lengths(c["T"], c["seqs"])) * D, "flops": 3.0 * n}
    n, q = c["T"] * c["kv_heads"] * D, c["T"] * H * D
    held = 2 if c["held"] == "bf16" else 1 + 1 / 32
    return {"bytes": 4.0 * q + 2 * (2 + held) * n
            + 4.0 * min(c["T"], max(_lengths(c["T"], c["seqs"]))) * D, "flops": 3.0 * (n + q)}


# ------------------------------------------------------- definitions, 64 bits
def _e4m3_64(v):
    """float64 v, |v| <= 448, to the nearest e4m3 value, ties to even."""
    e = torch.frexp(v)[1].double() - 1
    step = torch.exp2(e.clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _mx8_64(x):
    b = x.reshape(-1, 32)
    top = b.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448)).clamp(min=-127)
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e).clamp(min=-127)
    e = torch.where(top > 0, e, torch.zeros_like(e))
    return (_e4m3_64(b / torch.exp2(e)) * torch.exp2(e)).reshape(x.shape)


def _held_64(q, s):
    """float64 values of an MX8 tensor from its bits."""
    b = q.long()
    ex, man = (b >> 3) & 15, b & 7
    mag = torch.where(ex > 0, (8 + man).double() * torch.exp2(ex.double() - 10),
                      man.double() * 2.0 ** -9)
    v = torch.where(b >= 128, -mag, mag)
    return v * torch.exp2(s.double() - 127).repeat_interleave(32, -1)


def _rotated_64(x, cos, sin, interleaved):
    """As products of complex numbers."""
    x = x.double()
    pairs = x.unflatten(-1, (-1, 2)) if interleaved else x.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.complex(cos.double(), sin.double())[:, None]
    y = torch.view_as_real(z)
    return (y if interleaved else y.transpose(-1, -2)).flatten(-2)


def exact(case, seed):
    """The outputs in float64."""
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    d, D, H = torch.float64, case["dim"], case["heads"]
    if s["op"] == "prompt":
        T, g = s["T"], H // s["kv_heads"]
        q, k, v = (s[x].to(d).transpose(0, 1) for x in "QKV")
        out = {n: torch.zeros(x.shape, dtype=d, device="cuda") for n, x in
               ((("dQ", q), ("dK", k), ("dV", v)) if s["back"] else (("O", q),))}
        lse = torch.zeros((H, T), dtype=d, device="cuda")
        if s["back"]:
            do = s["dO"].to(d).transpose(0, 1)
        at = 0
        for n in s["lens"]:
            r = slice(at, at + n)
            at += n
            i = torch.arange(n, device="cuda")
            see = torch.ones((n, n), dtype=torch.bool, device="cuda")
            if s["causal"]:
                see &= i <= i[:, None]
            if s["window"]:
                see &= i[:, None] - i < s["window"]
            for h in range(H):
                z = s["scale"] * (q[h, r] @ k[h // g, r].T)
                z = z.masked_fill(~see, -torch.inf)
                lse[h, r] = torch.logsumexp(z, 1)
                p = torch.softmax(z, 1)
                if not s["back"]:
                    out["O"][h, r] = p @ v[h // g, r]
                    continue
                # o = p v, p = softmax(z): dz = p (dp - sum p dp)
                dp = do[h, r] @ v[h // g, r].T
                dz = s["scale"] * p * (dp - (p * dp).sum(1, keepdim=True))
                out["dV"][h // g, r] += p.T @ do[h, r]
                out["dQ"][h, r] = dz @ k[h // g, r]
                out["dK"][h // g, r] += dz.T @ q[h, r]
        out = {n: x.transpose(0, 1).contiguous() for n, x in out.items()}
        return out if s["back"] else {"O": out["O"], "lse": lse}
    if s["op"] == "decode":
        O = torch.empty(s["Q"].shape, dtype=d, device="cuda")
        g = H // s["kv_heads"]
        for b, n in enumerate(s["lens"]):
            t = torch.arange(max(0, n - s["window"]) if s["window"] else 0, n, device="cuda")
            page, row = s["table"][b, t // s["page"]].long(), t % s["page"]
            for h in range(s["kv_heads"]):
                k, v = (s["c" + x][page, h, row].to(d) if s["held"] == "bf16" else
                        _held_64(s["c" + x][page, h, row], s["c" + x + "s"][page, h, row])
                        for x in "kv")
                z = s["scale"] * (s["Q"][b, h * g:(h + 1) * g].to(d) @ k.T)
                O[b, h * g:(h + 1) * g] = torch.softmax(z, 1) @ v
        return {"O": O}
    at = torch.cat([torch.arange(n) for n in s["lens"]]).cuda() + s.get("past", 0)
    cos, sin = s["cos"][at], s["sin"][at]
    if s["op"] == "rope":
        return {"Y": _rotated_64(s["X"], cos, -sin if s["inverse"] else sin, s["interleaved"])}
    out = {"Q": _rotated_64(s["Q"], cos, sin, s["interleaved"])}
    new = {"k": _rotated_64(s["K"], cos, sin, s["interleaved"]), "v": s["V"].to(d)}
    first = 0
    for x in "kv":
        out[x] = s["c" + x].to(d) if s["held"] == "bf16" else _held_64(s["c" + x], s["c" + x + "s"])
    for b, n in enumerate(s["lens"]):
        for x in "kv":
            rows = new[x][first:first + n]
            rows = rows if s["held"] == "bf16" else _mx8_64(rows)
            t = at[first:first + n]
            out[x][s["table"][b, t // s["page"]].long(), :, t % s["page"]] = rows
        first += n
    return out
