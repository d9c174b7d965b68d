"""A Mixture-of-Experts block, served and trained, from the library's calls.

    python examples/moe_block.py                 # a decode batch, then a few training steps
    python examples/moe_block.py --tokens 1      # one sequence
    python examples/moe_block.py --bf16          # served with bf16 activations

`ServedBlock` is one block of an inference engine with its weights in MX4: the
attention's output projection, residual and norm, routing and the experts; the
activations of the experts are MX8 (or bf16), four library calls and the
router's product a step.  `TrainedBlock` is the block in training, forward and
gradients, in bf16.  All tensors a step writes are the block's own, made once.
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


def train(p, gating, tokens, steps, gen, lr=0.02):
    """Fits a fixed random map; returns the loss of every step."""
    p = {n: v for n, v in p.items() if n != "Wo"}
    block = TrainedBlock(**p, gating=gating, tokens=tokens)
    master = {n: p[n].float() for n in block.grads}
    X = torch.randn(tokens, p["w"].numel(), generator=gen, device="cuda").to(torch.bfloat16)
    want = torch.randn(X.shape, generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        diff = block.forward(X).float() - want
        losses.append(diff.square().mean().item())
        block.backward(X, (2 / tokens * diff).to(torch.bfloat16))
        for n, m in master.items():
            m -= lr * block.grads[n]
            p[n].copy_(m)
        block.balance()
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--tokens", type=int, default=64)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--hidden", type=int, default=2048)
    a.add_argument("--ffn", type=int, default=1408)
    a.add_argument("--experts", type=int, default=64)
    a.add_argument("--topk", type=int, default=6)
    a.add_argument("--bf16", action="store_true", help="bf16 activations in the served experts")
    a = a.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    gating = mf.make_gating(a.experts, a.topk, score="sigmoid", groups=4, top_groups=2, scale=2.5)
    p = weights(gen, a.hidden, a.ffn, a.experts, a.hidden)
    ms = serve(p, gating, a.tokens, a.steps, not a.bf16, gen)
    print(f"served: {a.tokens} tokens, {'bf16' if a.bf16 else 'MX8'} activations, {ms * 1e3:.0f} us a step")
    losses = train(p, gating, max(a.tokens, 256), a.steps, gen)
    print(f"trained: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")


if __name__ == "__main__":
    main()
