"""A Mixture-of-Experts block, served and trained, from the library's calls.

    python examples/moe_block.py                 # a decode batch, then a few training steps
    python examples/moe_block.py --tokens 1      # one sequence
    python examples/moe_block.py --bf16          # served with bf16 activations
    python examples/moe_block.py --context 8000  # after sequences of 8000 tokens

`ServedAttention` stands in front of a block of an inference engine: the projection
of queries, keys and values, their rotation, the cache of pages (MX8, or bf16) and the
attention over it, for whole prompts and then token by token; `TrainedAttention` is
the same in training, over packed sequences.  `ServedBlock` is one block of an
inference engine with its weights in MX4: the attention's output projection, residual
and norm, routing and the experts; the activations of the experts are MX8 (or bf16),
four library calls and the router's product a step.  `TrainedBlock` is the block in
training, forward and gradients, in bf16.  `ServedLayer` and `TrainedLayer` join
attention and block.  What a step of a block writes are the block's own tensors, made once.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2511_21431_amd as mf  # noqa: E402

EPS = 1e-6


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def tables(positions, dim, base=10000.0):
    """Cosines and sines of the rotation, float [positions, dim / 2]."""
    f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cos(a).float(), torch.sin(a).float()


def offsets_of(lens):
    return torch.tensor([0, *lens], device="cuda").cumsum(0).to(torch.int32)


class ServedAttention:
    """Wqkv [(heads + 2 kv_heads) dim, h]: rounded to MX4 once, here.  The cache holds
    `sequences` of up to `positions` tokens; each has the same pages for good."""

    def __init__(self, Wqkv, attn, sequences, positions, page=64, mx8=True):
        self.attn, self.H, self.Hk, self.D = attn, attn.heads, attn.kv_heads, attn.dim
        self.N, self.h = Wqkv.shape
        self.W = mf.memfine_mxw_quantize(Wqkv[None])
        self.cos, self.sin = tables(positions, self.D)
        width = -(-positions // page)
        size = (sequences * width, self.Hk, page, self.D)
        if mx8:
            kv = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
            kv += [torch.zeros((*size[:3], self.D // 32), dtype=torch.uint8, device="cuda")
                   for _ in range(2)]
        else:
            kv = [torch.zeros(size, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.cache = mf.make_cache(*kv)
        self.table = torch.arange(sequences * width, dtype=torch.int32, device="cuda").view(sequences, width)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.qkv, self.q, self.out = (empty(sequences, n) for n in (self.N, self.H * self.D, self.H * self.D))

    def split(self, qkv):
        x = qkv.view(-1, self.H + 2 * self.Hk, self.D)
        return x[:, :self.H], x[:, self.H:self.H + self.Hk], x[:, self.H + self.Hk:]

    def prompt(self, x, lens):
        """Rows x [sum(lens), h] of one new prompt a sequence; returns [sum(lens), H D]."""
        offsets = offsets_of(lens)
        self.lengths.copy_(offsets[1:] - offsets[:-1])
        qkv, turned, out = (empty(len(x), n) for n in (self.N, self.H * self.D, self.H * self.D))
        mf.memfine_linear_mxw(self.N, self.h, x, *self.W, qkv)
        q, k, v = self.split(qkv)
        turned, out = turned.view(q.shape), out.view(q.shape)
        # (keys go into the cache unrounded, like those of later tokens; as rows they are turned
        # for the prompts' own attention)
        mf.memfine_kv_write(self.cache, self.table, self.lengths, k, v, offsets=offsets, Q=q, R=turned,
                            cos=self.cos, sin=self.sin)
        mf.memfine_rope(offsets, self.cos, self.sin, k, k)
        mf.memfine_attn_fwd(self.attn, offsets, turned, k, v, out)
        return out.view(len(x), -1)

    def step(self, x, allocator=None):
        """Rows x [sequences, h] of one new token a sequence; returns [sequences, H D]."""
        self.lengths += 1
        mf.memfine_linear_mxw(self.N, self.h, x, *self.W, self.qkv, allocator=allocator)
        q, k, v = self.split(self.qkv)
        shape = (len(x), self.H, self.D)
        mf.memfine_kv_write(self.cache, self.table, self.lengths, k, v, Q=q, R=self.q.view(shape),
                            cos=self.cos, sin=self.sin)
        mf.memfine_attn_decode(self.attn, self.cache, self.table, self.lengths, self.q.view(shape),
                               self.out.view(shape), allocator=allocator)
        return self.out


class TrainedAttention:
    """out = attention(X Wqkv^T) Wo^T over packed sequences of lengths `lens`; the
    gradients of both weights are float tensors."""

    def __init__(self, Wqkv, Wo, attn, lens):
        self.Wqkv, self.Wo, self.attn, self.offsets = Wqkv, Wo, attn, offsets_of(lens)
        H, Hk, D, T = attn.heads, attn.kv_heads, attn.dim, sum(lens)
        self.H, self.both = H, H + Hk
        self.cos, self.sin = tables(max(lens), D)
        self.qkv, self.dqkv = (empty(T, H + 2 * Hk, D) for _ in range(2))
        self.o, self.lse = empty(T, H, D), empty(H, T, dtype=torch.float32)
        self.grads = {n: torch.zeros_like(p, dtype=torch.float32) for n, p in (("Wqkv", Wqkv), ("Wo", Wo))}

    def split(self, x):
        return x[:, :self.H], x[:, self.H:self.both], x[:, self.both:]

    def forward(self, X):
        torch.matmul(X, self.Wqkv.t(), out=self.qkv.view(len(X), -1))
        turned = self.qkv[:, :self.both]
        mf.memfine_rope(self.offsets, self.cos, self.sin, turned, turned)
        mf.memfine_attn_fwd(self.attn, self.offsets, *self.split(self.qkv), self.o, self.lse)
        return self.o.view(len(X), -1) @ self.Wo.t()

    def backward(self, X, dout):
        """dX of the last forward's X; the weights' gradients are overwritten."""
        T = len(X)
        self.grads["Wo"].copy_(dout.t() @ self.o.view(T, -1))
        do = (dout @ self.Wo).view(self.o.shape)
        mf.memfine_attn_bwd(self.attn, self.offsets, *self.split(self.qkv), self.o, self.lse, do,
                            *self.split(self.dqkv))
        turned = self.dqkv[:, :self.both]
        mf.memfine_rope(self.offsets, self.cos, self.sin, turned, turned, inverse=True)
        d = self.dqkv.view(T, -1)
        self.grads["Wqkv"].copy_(d.t() @ X)
        return d @ self.Wqkv


class ServedBlock:
    """Wo [h, K], W1 [E, 2F, h], W2 [E, h, F]: rounded to MX4 once, here.  Wr
    [E, h] and the norm's weight w [h] stay bf16; bias float [E] balances the
    selection."""

    def __init__(self, Wo, w, Wr, bias, W1, W2, gating, tokens, mx8=True):
        self.h, self.K = Wo.shape
        self.E, self.F = W1.shape[0], W2.shape[2]
        self.w, self.Wr, self.bias, self.gating = w, Wr, bias, gating
        self.Wo = mf.memfine_mxw_quantize(Wo[None])
        self.W1, self.W2 = mf.memfine_mxw_quantize(W1), mf.memfine_mxw_quantize(W2)
        self.shape = mf.make_shape(tokens, self.h, self.F, self.E, gating.k, mf.BF16)
        self.o, self.y, self.out = (empty(tokens, self.h) for _ in range(3))
        self.q = empty(tokens, self.h, dtype=torch.uint8) if mx8 else None
        self.qs = empty(tokens, self.h // 32, dtype=torch.uint8) if mx8 else None
        self.logits = empty(tokens, self.E, dtype=torch.float32)
        self.idx = empty(tokens, gating.k, dtype=torch.int32)
        self.gates = empty(tokens, gating.k, dtype=torch.float32)

    def step(self, attended, stream, allocator=None):
        """attended [tokens, K]: the heads' outputs; stream [tokens, h]: the
        residual stream, to which the projection is added in place.  Returns the
        experts' output, which the next block adds.  allocator: working memory of
        the caller's, for steps captured into a graph (without one each capture
        keeps memory of the library's until the process ends); it serves one
        request at a time, memfine_moe_mxw_workspace_bytes or
        memfine_linear_mxw_workspace_bytes, whichever is more."""
        mf.memfine_linear_mxw(self.h, self.K, attended, *self.Wo, self.o, allocator=allocator)
        mf.memfine_norm_fwd(EPS, self.o, self.w, R=stream, S=stream, Y=self.y, Q=self.q, QS=self.qs)
        mf.memfine_router_logits(self.shape, self.y, self.Wr, self.logits)
        mf.memfine_route_fwd(self.gating, self.logits, self.idx, self.gates, bias=self.bias)
        mf.memfine_moe_fwd_mxw(self.shape, 1, self.y if self.q is None else self.q, self.idx,
                               self.gates, *self.W1, *self.W2, self.out, XS=self.qs,
                               allocator=allocator)
        return self.out


class TrainedBlock:
    """out = experts(norm(X)) + X with routing from logits; the gradients of all
    weights are summed into float tensors."""

    def __init__(self, w, Wr, bias, W1, W2, gating, tokens, chunks=1):
        self.w, self.Wr, self.bias, self.W1, self.W2 = w, Wr, bias, W1, W2
        self.gating, self.chunks = gating, chunks
        E, h, F = W2.shape
        self.shape = mf.make_shape(tokens, h, F, E, gating.k, mf.BF16)
        self.y, self.out, self.dy, self.dX = (empty(tokens, h) for _ in range(4))
        self.logits, self.dlogits = (empty(tokens, E, dtype=torch.float32) for _ in range(2))
        self.idx = empty(tokens, gating.k, dtype=torch.int32)
        self.gates, self.dgates = (empty(tokens, gating.k, dtype=torch.float32) for _ in range(2))
        self.grads = {n: torch.zeros_like(p, dtype=torch.float32)
                      for n, p in (("w", w), ("Wr", Wr), ("W1", W1), ("W2", W2))}

    def forward(self, X):
        mf.memfine_norm_fwd(EPS, X, self.w, Y=self.y)
        mf.memfine_router_logits(self.shape, self.y, self.Wr, self.logits)
        mf.memfine_route_fwd(self.gating, self.logits, self.idx, self.gates, bias=self.bias)
        mf.memfine_moe_fwd(self.shape, self.chunks, self.y, self.idx, self.gates, self.W1, self.W2,
                           self.out)
        return self.out + X

    def backward(self, X, dout):
        """dX of the last forward's X; the weights' gradients are overwritten."""
        g = self.grads
        mf.memfine_moe_bwd(self.shape, self.chunks, self.y, self.idx, self.gates, self.W1, self.W2,
                           dout, self.dy, g["W1"], g["W2"], self.dgates)
        mf.memfine_route_bwd(self.gating, self.logits, self.idx, self.dgates, self.dlogits)
        mf.memfine_router_logits_bwd(self.shape, self.y, self.Wr, self.dlogits, self.dy, g["Wr"],
                                     accumulate_dX=True)
        mf.memfine_norm_bwd(EPS, X, self.w, self.dy, self.dX, g["w"], dS=dout)
        return self.dX

    def balance(self, rate=1e-3):
        """Moves the selection's bias towards experts with fewer tokens than the mean."""
        load = torch.bincount(self.idx.reshape(-1), minlength=self.gating.E).float()
        self.bias += rate * torch.sign(load.mean() - load)


class ServedLayer:
    """A decode step of norm, attention and block; w [h]: weight of the norm in front of the
    attention."""

    def __init__(self, w, attention, block):
        self.w, self.attention, self.block = w, attention, block
        self.y = empty(block.o.shape[0], block.h)

    def step(self, added, stream, allocator=None):
        """added [tokens, h]: what the layer before this one adds to the residual stream
        [tokens, h], which is updated in place.  Returns what the next one adds."""
        mf.memfine_norm_fwd(EPS, added, self.w, R=stream, S=stream, Y=self.y)
        return self.block.step(self.attention.step(self.y, allocator), stream, allocator)


class TrainedLayer:
    """out = block(X + attention(X))."""

    def __init__(self, attention, block):
        self.attention, self.block = attention, block
        self.grads = {**attention.grads, **block.grads}

    def forward(self, X):
        self.x = X + self.attention.forward(X)
        return self.block.forward(self.x)

    def backward(self, X, dout):
        d = self.block.backward(self.x, dout)
        return d + self.attention.backward(X, d)

    def balance(self, rate=1e-3):
        self.block.balance(rate)


def weights(gen, h, F, E, K):
    def normal(*shape, std):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(torch.bfloat16)
    return dict(Wo=normal(h, K, std=K ** -0.5), w=normal(h, std=0.1) + 1, Wr=normal(E, h, std=h ** -0.5),
                bias=torch.zeros(E, device="cuda"), W1=normal(E, 2 * F, h, std=h ** -0.5),
                W2=normal(E, h, F, std=F ** -0.5))


def serve(p, gating, tokens, steps, mx8, gen):
    block = ServedBlock(**p, gating=gating, tokens=tokens, mx8=mx8)
    attended = torch.randn(tokens, block.K, generator=gen, device="cuda").to(torch.bfloat16)
    stream = torch.randn(tokens, block.h, generator=gen, device="cuda").to(torch.bfloat16)
    for _ in range(3):
        block.step(attended, stream.clone())
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(steps):
        block.step(attended, stream)
    stop.record()
    stop.synchronize()
    return start.elapsed_time(stop) / steps


def qkv_weight(gen, attn, h):
    n = (attn.heads + 2 * attn.kv_heads) * attn.dim
    return (torch.randn(n, h, generator=gen, device="cuda") * h ** -0.5).to(torch.bfloat16)


def serve_layer(p, gating, attn, tokens, context, steps, mx8, gen):
    """Milliseconds a step of attention and block, for `tokens` sequences that have `context`
    tokens each."""
    h = p["w"].numel()
    a = ServedAttention(qkv_weight(gen, attn, h), attn, tokens, context + steps + 3)
    layer = ServedLayer(torch.ones_like(p["w"]), a, ServedBlock(**p, gating=gating, tokens=tokens, mx8=mx8))
    stream = torch.randn(tokens, h, generator=gen, device="cuda").to(torch.bfloat16)
    a.prompt(stream.repeat_interleave(context, 0), [context] * tokens)
    added = torch.zeros_like(stream)
    for _ in range(3):
        added = layer.step(added, stream)
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(steps):
        added = layer.step(added, stream)
    stop.record()
    stop.synchronize()
    return start.elapsed_time(stop) / steps


def train(p, gating, tokens, steps, gen, lr=0.02, attn=None):
    """Fits a fixed random map; returns the loss of every step.  With attn the layer
    begins with attention over three sequences, which the tokens are split into."""
    Wo, p = p["Wo"], {n: v for n, v in p.items() if n != "Wo"}
    layer = TrainedBlock(**p, gating=gating, tokens=tokens)
    if attn is not None:
        lens = [tokens // 2, tokens // 3]
        p["Wqkv"], p["Wo"] = qkv_weight(gen, attn, p["w"].numel()), Wo
        layer = TrainedLayer(TrainedAttention(p["Wqkv"], Wo, attn, [*lens, tokens - sum(lens)]), layer)
    master = {n: p[n].float() for n in layer.grads}
    X = torch.randn(tokens, p["w"].numel(), generator=gen, device="cuda").to(torch.bfloat16)
    want = torch.randn(X.shape, generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        diff = layer.forward(X).float() - want
        losses.append(diff.square().mean().item())
        layer.backward(X, (2 / tokens * diff).to(torch.bfloat16))
        for n, m in master.items():
            g = layer.grads[n]
            # (the attention has no norm in front: its weights move by 1 % of theirs at most)
            m -= g * (torch.clamp(0.01 * m.norm() / g.norm(), max=lr) if n in ("Wqkv", "Wo") else lr)
            p[n].copy_(m)
        layer.balance()
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--tokens", type=int, default=64)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--hidden", type=int, default=2048)
    a.add_argument("--ffn", type=int, default=1408)
    a.add_argument("--experts", type=int, default=64)
    a.add_argument("--topk", type=int, default=6)
    a.add_argument("--heads", type=int, default=16)
    a.add_argument("--kv-heads", type=int, default=4)
    a.add_argument("--context", type=int, default=1000, help="tokens of each sequence before the step")
    a.add_argument("--bf16", action="store_true", help="bf16 activations in the served experts")
    a = a.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    gating = mf.make_gating(a.experts, a.topk, score="sigmoid", groups=4, top_groups=2, scale=2.5)
    attn = mf.make_attn(a.heads, a.kv_heads, 128)
    p = weights(gen, a.hidden, a.ffn, a.experts, attn.heads * attn.dim)
    ms = serve(p, gating, a.tokens, a.steps, not a.bf16, gen)
    print(f"served: {a.tokens} tokens, {'bf16' if a.bf16 else 'MX8'} activations, {ms * 1e3:.0f} us a step")
    ms = serve_layer(p, gating, attn, a.tokens, a.context, a.steps, not a.bf16, gen)
    print(f"with attention: {a.tokens} sequences of {a.context} tokens, MX8 cache, {ms * 1e3:.0f} us a step")
    losses = train(p, gating, max(a.tokens, 256), a.steps, gen, attn=attn)
    print(f"trained: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")


if __name__ == "__main__":
    main()
