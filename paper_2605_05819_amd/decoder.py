"""A decoder layer of compensated quantized linears, from the library's calls:

    q, k, v = window(n)                        cl.linear_decode_window / linear_prefill
    q       = rotated, k and v to the cache    cl.kv_append
    a       = attention over the cache         cl.attention
    h, n    = h + o(a), norm                   cl.linear_*, cl.residual_norm
    y       = down(SiLU(gate n) * up n)        cl.linear_decode_glu, cl.linear_decode    (dense)
    y       = down_e(SiLU(gate_e n) * up_e n)  cl.moe_route, cl.moe_linear_decode_*      (experts)
    h, n    = h + y (or its weighted slots), the next layer's norm

``h`` is the residual stream and ``n`` its normalised value, both [tokens][hidden];
a step takes the pair and returns the next layer's.  Up to 64 tokens go through
the decode calls, more (dense layers only) through the prefill ones.

    python -m paper_2605_05819_amd.decoder

runs a few layers of random weights over a prompt and some decode steps, and
prints the times.
"""

import time
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import cl

DECODE_TOKENS = 64          # most tokens of the decode and MoE calls


@dataclass
class Linear:
    """A compensated linear: its packed backbone and factors (or None)."""
    w: cl.QWeight
    c: Optional[cl.LowRank] = None


def linear(lin, x, out_dtype):
    """``lin`` on [tokens][d_in], by the decode call or the prefill one."""
    call = cl.linear_decode if x.shape[0] <= DECODE_TOKENS else cl.linear_prefill
    return call(lin.w, lin.c, x, out_dtype)


def window(lins, x, out_dtype):
    """Linears that share x: one window where the decode calls reach."""
    if x.shape[0] <= DECODE_TOKENS:
        return cl.linear_decode_window([p.w for p in lins], [p.c for p in lins], x, out_dtype)
    return [cl.linear_prefill(p.w, p.c, x, out_dtype) for p in lins]


@dataclass
class Dense:
    """The gated MLP of a dense layer."""
    gate: Linear
    up: Linear
    down: Linear

    def __call__(self, n):
        if n.shape[0] <= DECODE_TOKENS:
            g = cl.linear_decode_glu([self.gate.w, self.up.w], [self.gate.c, self.up.c], n, n.dtype)
        else:
            # fp32 as in the decode call's epilogue: one rounding, of the product (a
            # 2048-token block of 14336 takes 886 us so, 833 with g and u in 16 bits)
            g, u = window([self.gate, self.up], n, torch.float32)
            g = torch.mul(torch.nn.functional.silu(g, inplace=True), u, out=torch.empty_like(g, dtype=n.dtype))
        return linear(self.down, g, n.dtype), None


@dataclass
class Experts:
    """The routed experts of a MoE layer.  ``router`` [experts][hidden] is the
    (unquantized) routing weight in the activations' dtype; its logits stay in
    fp32, since 16 bits would tie many and decide those by the lower id.  With
    ``levels`` the slots' ranks follow their routing weights (the
    expert-activation term)."""
    router: torch.Tensor
    rule: cl.Router
    gate: cl.MoeExperts
    up: cl.MoeExperts
    down: cl.MoeExperts
    levels: Sequence[int] = ()

    def __call__(self, n):
        if n.shape[0] > DECODE_TOKENS:
            raise ValueError("a MoE layer takes at most %d tokens a step" % DECODE_TOKENS)
        logits = torch.mm(n, self.router.t(), out_dtype=torch.float32)
        projections = (self.gate, self.up, self.down)
        if self.levels:
            ids, weights, ranks = cl.moe_route(self.rule, logits, [p.ranks for p in projections], self.levels)
        else:
            (ids, weights), ranks = cl.moe_route(self.rule, logits), [None] * 3
        g, u = cl.moe_linear_decode_window([self.gate, self.up], n, ids, n.dtype, slot_ranks=ranks[:2])
        return cl.moe_linear_decode_gated(self.down, g, u, ids, n.dtype, slot_ranks=ranks[2]), weights


@dataclass
class DecoderLayer:
    """One layer: Q/K/V and O, the block behind them and their norms (weights
    in the activations' dtype).  q_norm and k_norm: per-head norms, or None."""
    q: Linear
    k: Linear
    v: Linear
    o: Linear
    block: object                       # Dense or Experts
    rope: cl.Rope
    q_heads: int
    block_norm: torch.Tensor
    q_norm: Optional[torch.Tensor] = None
    k_norm: Optional[torch.Tensor] = None
    eps: float = 1e-6
    attn_window: int = 0

    def step(self, h, n, cache, batch, next_norm):
        """(h, n) of this layer's new tokens -> (h, n) for the next layer,
        whose norm weight is ``next_norm``; their keys and values go to
        ``cache`` (this layer's) where ``batch`` says."""
        T, dt = n.shape[0], n.dtype
        q, k, v = window([self.q, self.k, self.v], n, dt)
        q, k, v = (x.view(T, heads, cache.head_dim) for x, heads in
                   ((q, self.q_heads), (k, cache.kv_heads), (v, cache.kv_heads)))
        q = cl.kv_append(cache, batch, k, v, q=q, rope=self.rope, q_norm=self.q_norm, k_norm=self.k_norm,
                         eps=self.eps, q_out=q)
        a = cl.attention(cache, batch, q, window=self.attn_window)
        h, n = cl.residual_norm(linear(self.o, a.view(T, -1), dt), self.block_norm, residual=h, eps=self.eps)
        y, weights = self.block(n)
        return cl.residual_norm(y, next_norm, residual=h, slot_weights=weights, eps=self.eps)


def run(layers, caches, batch, x, norms, last_norm, eps=1e-6):
    """The layers over the new tokens' embeddings x [tokens][hidden]; norms:
    the weight ahead of each layer's Q/K/V, last_norm the one behind the last
    layer.  Returns (residual stream, its last norm)."""
    h, n = x, cl.residual_norm(x, norms[0], eps=eps, h=False)
    for layer, cache, nxt in zip(layers, caches, [*norms[1:], last_norm]):
        h, n = layer.step(h, n, cache, batch, nxt)
    return h, n


# ------------------------------------------------------------------ the example

def _random_linear(g, d_out, d_in, rank=32, dev="cuda"):
    W = torch.randn((d_out, d_in), generator=g, device=dev) * 0.02
    A = (torch.randn((rank, d_in), generator=g, device=dev) * 0.01).half()
    B = (torch.randn((d_out, rank), generator=g, device=dev) * 0.01).half()
    return Linear(cl.quantize_pack(W, 4, 128), cl.LowRank(A, B, rank, rank))


def random_dense_layer(g, hidden=4096, kv=1024, ffn=14336, head_dim=128, dtype=torch.float16, dev="cuda"):
    """A Llama-3.1-8B-shaped layer of random weights."""
    mk = lambda o, i: _random_linear(g, o, i, dev=dev)  # noqa: E731
    freq, mag = cl.rope_frequencies(head_dim, 500000.0, "bands", 8.0, 8192, 1.0, 4.0)
    return DecoderLayer(mk(hidden, hidden), mk(kv, hidden), mk(kv, hidden), mk(hidden, hidden),
                        Dense(mk(ffn, hidden), mk(ffn, hidden), mk(hidden, ffn)), cl.Rope(freq.to(dev), magnitude=mag),
                        hidden // head_dim, torch.ones(hidden, dtype=dtype, device=dev))


def main(layers=4, seqs=8, prompt=256, steps=16, page=64):
    dev, dt, hidden, kv_heads, head_dim = "cuda", torch.float16, 4096, 8, 128
    g = torch.Generator(device=dev).manual_seed(0)
    stack = [random_dense_layer(g, dtype=dt) for _ in range(layers)]
    norms = [torch.ones(hidden, dtype=dt, device=dev) for _ in range(layers + 1)]
    width = -(-(prompt + steps) // page)
    caches = [cl.KvCache.empty(seqs * width, page, kv_heads, head_dim, dt, dev) for _ in stack]
    table = torch.randperm(seqs * width, generator=g, device=dev).to(torch.int32).view(seqs, width)
    kv_len = torch.full((seqs,), prompt, dtype=torch.int32, device=dev)
    batch = cl.KvBatch(kv_len, table, seqs * prompt, q_len=prompt, max_kv_len=prompt + steps)
    x = torch.randn((seqs * prompt, hidden), generator=g, device=dev).to(dt)
    for _ in range(2):
        torch.cuda.synchronize()
        t = time.perf_counter()
        run(stack, caches, batch, x, norms[:-1], norms[-1])
        torch.cuda.synchronize()
        first = time.perf_counter() - t
    print("prompt: %d x %d tokens, %d layers, %.1f ms" % (seqs, prompt, layers, first * 1e3))
    # the decode step, captured once and replayed for every token
    batch = cl.KvBatch(kv_len, table, seqs, max_kv_len=prompt + steps)
    x = torch.randn((seqs, hidden), generator=g, device=dev).to(dt)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv_len.add_(1)
        run(stack, caches, batch, x, norms[:-1], norms[-1])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(stack, caches, batch, x, norms[:-1], norms[-1])
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps - 1):
        kv_len.add_(1)
        graph.replay()
    torch.cuda.synchronize()
    print("decode: %d sequences, %.1f us a layer and token" % (seqs, (time.perf_counter() - t) / (steps - 1) / layers * 1e6))


if __name__ == "__main__":
    main()
