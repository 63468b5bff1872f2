"""A decoder layer's step through all of its calls, against the fp64 oracle's
composition of the same layer: prompts, then decode steps over the cache they
left, dense and with routed experts, eagerly and from a captured graph.

Each of the step's seven calls is held to a relative L2 of 1e-3 by its own tests
(fp16 values between them); the norms keep relative errors as they are and the
gated product adds two, so the composed outputs are held to 1e-2."""

import numpy as np
import pytest
import torch

from oracle import layer as ol, linear as olin, moe as omoe, quant
from paper_2605_05819_amd import cl, decoder, workloads as wl
from tests.helpers import dev_f16, dev_u32, oracle_layer, rel_l2

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HKV, D, FFN, PAGE = 256, 4, 2, 64, 512, 16


def _linear(d_out, d_in, seed, rank=8):
    Q, s, z, A, B, _ = oracle_layer(wl.weight((d_out, d_in), seed, std=0.05), 4, 128, rank)
    w = cl.QWeight(dev_u32(Q), dev_f16(s), dev_f16(z), d_out, d_in, 4, 128)
    return (decoder.Linear(w, cl.LowRank(dev_f16(A), dev_f16(B), rank, rank)),
            (quant.dequant_packed(Q, s, z, 4, 128, d_in), A, B, rank))


def _experts(E, d_out, d_in, seed, r_max=8):
    parts = [oracle_layer(wl.weight((d_out, d_in), seed, 0, 0, e, std=0.05), 4, 128, r_max)[:5] for e in range(E)]
    Q, s, z, A, B = (np.stack([p[i] for p in parts]) for i in range(5))
    ranks = np.full(E, r_max, np.int32)
    ex = cl.MoeExperts(dev_u32(Q), dev_f16(s), dev_f16(z), dev_f16(A), dev_f16(B), torch.from_numpy(ranks).cuda(), E, d_out,
                       d_in, 4, 128, r_max)
    return ex, [(quant.dequant_packed(p[0], p[1], p[2], 4, 128, d_in), p[3], p[4]) for p in parts], ranks


class Layer:
    """The device layer and the oracle's, with the oracle's own (unpaged) cache."""

    def __init__(self, moe, seqs, seed=3):
        g = np.random.default_rng(seed)
        norm = lambda n: dev_f16(1 + 0.1 * g.standard_normal(n))  # noqa: E731
        dev, self.o = {}, {}
        for i, (name, shape) in enumerate(dict(q=(HQ * D, HIDDEN), k=(HKV * D, HIDDEN), v=(HKV * D, HIDDEN),
                                               o=(HIDDEN, HQ * D)).items()):
            dev[name], self.o[name] = _linear(*shape, 100 + i)
        self.norms = [norm(HIDDEN) for _ in range(3)]          # before attention, before the block, behind it
        self.qn, self.kn = norm(D), norm(D)
        freq, _ = cl.rope_frequencies(D, 10000.0)
        self.freq = freq.double().numpy()
        self.moe = moe
        if moe:
            E, k = 8, 3
            self.router = dev_f16(g.standard_normal((E, HIDDEN)) * 0.3)
            gate, self.og, self.ranks = _experts(E, FFN, HIDDEN, 200)
            up, self.ou, _ = _experts(E, FFN, HIDDEN, 201)
            down, self.od, _ = _experts(E, HIDDEN, FFN, 202)
            block = decoder.Experts(self.router, cl.Router(E, k), gate, up, down, levels=(0, 4, 8))
        else:
            ls = [_linear(FFN, HIDDEN, 200), _linear(FFN, HIDDEN, 201), _linear(HIDDEN, FFN, 202)]
            block = decoder.Dense(*[p[0] for p in ls])
            self.og, self.ou, self.od = [p[1] for p in ls]
        self.dev = decoder.DecoderLayer(**dev, block=block, rope=cl.Rope(freq.cuda()), q_heads=HQ,
                                        block_norm=self.norms[1], q_norm=self.qn, k_norm=self.kn)
        self.keys = [np.zeros((HKV, 0, D)) for _ in range(seqs)]
        self.values = [np.zeros((HKV, 0, D)) for _ in range(seqs)]

    def lin(self, p, x):
        return olin.forward(*p, x)

    def oracle(self, x, counts):
        """x [tokens][HIDDEN] fp64, counts new tokens of each sequence -> (h, n)."""
        w = [t.double().cpu().numpy() for t in self.norms]
        n = ol.normalise(x, "rms", 1e-6) * w[0]
        q, k, v = (self.lin(self.o[i], n).reshape(len(x), -1, D) for i in "qkv")
        a, at = np.zeros_like(q), 0
        for b, c in enumerate(counts):
            base = self.keys[b].shape[1]
            for j in range(c):
                t = at + j
                q[t] = ol.rotate(ol.head_norm(q[t], self.qn.double().cpu().numpy(), 1e-6), base + j, self.freq)
                kk = ol.rotate(ol.head_norm(k[t], self.kn.double().cpu().numpy(), 1e-6), base + j, self.freq)
                self.keys[b] = np.concatenate([self.keys[b], kk[:, None]], 1)
                self.values[b] = np.concatenate([self.values[b], v[t][:, None]], 1)
            if c:
                a[at:at + c] = ol.attend(q[at:at + c], self.keys[b], self.values[b], D ** -0.5)[0]
            at += c
        h, n = ol.residual_norm(self.lin(self.o["o"], a.reshape(len(x), -1)), w[1], residual=x)
        if not self.moe:
            y = self.lin(self.od, olin.silu(self.lin(self.og, n)) * self.lin(self.ou, n))
            return ol.residual_norm(y, w[2], residual=h)
        ids, g, _ = ol.route(n @ self.router.double().cpu().numpy().T, 3)
        ranks = np.minimum(wl.dynamic_slot_ranks(ids, g, self.ranks, (0, 4, 8), 8), 8)
        up = [omoe.forward(p, self.ranks, n, ids, False, slot_ranks=ranks) for p in (self.og, self.ou)]
        y = omoe.forward(self.od, self.ranks, olin.silu(up[0]) * up[1], ids, True, slot_ranks=ranks)
        return ol.residual_norm(y, w[2], residual=h, slot_weights=g)


def _batch(kv_len, table, counts, most):
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return cl.KvBatch(kv_len, table, int(start[-1]), q_len=max(counts), q_start=torch.from_numpy(start).cuda(), max_kv_len=most)


@pytest.mark.parametrize("moe", [False, True], ids=["dense", "experts"])
def test_layer_steps_against_oracle(moe):
    seqs, most = 3, 80
    L = Layer(moe, seqs)
    width = -(-most // PAGE)
    cache = cl.KvCache.empty(seqs * width + 1, PAGE, HKV, D)
    table = torch.randperm(seqs * width + 1)[:seqs * width].view(seqs, width).to(torch.int32).cuda()
    g = np.random.default_rng(9)
    total = np.zeros(seqs, np.int32)
    # prompts (over 64 tokens in all takes the prefill calls), decode, a mixed step
    for counts in ([17, 1, 30] if moe else [17, 1, 60], [1, 1, 1], [1, 5, 0], [2, 1, 1]):
        total += np.asarray(counts, np.int32)
        x = g.standard_normal((sum(counts), HIDDEN)).astype(np.float16)
        batch = _batch(torch.from_numpy(total.copy()).cuda(), table, counts, most)
        xd = torch.from_numpy(x).cuda()
        h, n = decoder.run([L.dev], [cache], batch, xd, L.norms[:1], L.norms[2])
        torch.cuda.synchronize()
        rh, rn = L.oracle(x.astype(np.float64), counts)
        assert rel_l2(h.double().cpu().numpy(), rh) <= 1e-2 and rel_l2(n.double().cpu().numpy(), rn) <= 1e-2


@pytest.mark.parametrize("moe", [False, True], ids=["dense", "experts"])
def test_captured_decode_step_replays_like_the_eager_one(moe):
    """The step captured once; kv_len moves on in place between the replays, with eager work and
    synchronizations among them.  Every replay equals the eager step bit for bit."""
    seqs, most = 4, 64
    L = Layer(moe, seqs)
    width = -(-most // PAGE)
    caches = [cl.KvCache.empty(seqs * width, PAGE, HKV, D) for _ in range(2)]
    table = torch.arange(seqs * width, dtype=torch.int32).view(seqs, width).cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    for c in caches:
        c.k.copy_(torch.randn(c.k.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)))
        c.v.copy_(torch.randn(c.v.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)))
    kv_len = torch.tensor([5, 17, 1, 40], dtype=torch.int32, device="cuda")
    batch = cl.KvBatch(kv_len, table, seqs, max_kv_len=most)
    x = torch.randn((seqs, HIDDEN), device="cuda", generator=g).half()
    step = lambda c: decoder.run([L.dev], [c], batch, x, L.norms[:1], L.norms[2])  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in caches:
            step(c)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0])
    for _ in range(4):
        kv_len.add_(1)
        x.copy_(torch.randn((seqs, HIDDEN), device="cuda", generator=g))
        want = step(caches[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert all(torch.equal(a, b) for a, b in ((caches[0].k, caches[1].k), (caches[0].v, caches[1].v)))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
def test_experts_are_chosen_by_unrounded_logits(dtype):
    """Logits of 64 and 64 + 2^-6, which 16 bits cannot tell apart: the larger one decides, not the lower id."""
    E, hidden, ffn = 8, 256, 128
    router = torch.zeros((E, hidden))
    router[2], router[5] = 0.25, 0.25
    router[5, 17] += 2.0 ** -6
    gate, og, ranks = _experts(E, ffn, hidden, 300)
    up, ou, _ = _experts(E, ffn, hidden, 301)
    down, od, _ = _experts(E, hidden, ffn, 302)
    block = decoder.Experts(router.to(dtype).cuda(), cl.Router(E, 1), gate, up, down)
    n = torch.ones((3, hidden), dtype=dtype, device="cuda")
    y, w = block(n)
    torch.cuda.synchronize()
    ids = np.full((3, 1), 5)
    g, u = (omoe.forward(p, ranks, n.double().cpu().numpy(), ids, False) for p in (og, ou))
    want = omoe.forward(od, ranks, olin.silu(g) * u, ids, True)
    assert rel_l2(y.double().cpu().numpy(), want) <= 1e-2 and (w == 1).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("tokens", [65, 200])
def test_gated_activation_is_rounded_once(tokens, dtype, monkeypatch):
    """SiLU(g) u of a prompt, as the decode call does: one rounding of the fp32 value (2^-20 of it for fp32 itself)."""
    ls = [_linear(FFN, HIDDEN, 200)[0], _linear(FFN, HIDDEN, 201)[0]]
    x = torch.from_numpy(np.random.default_rng(4).standard_normal((tokens, HIDDEN))).to(dtype).cuda()
    monkeypatch.setattr(decoder, "linear", lambda lin, a, out_dtype: a)
    got, none = decoder.Dense(*ls, None)(x)
    g, u = (t.double() for t in decoder.window(ls, x, torch.float32))
    torch.cuda.synchronize()
    want = g / (1 + torch.exp(-g)) * u
    u16 = 2.0 ** (-11 if dtype == torch.float16 else -8)
    assert none is None and got.dtype == dtype
    assert ((got.double() - want).abs() <= (u16 + 2.0 ** -20) * want.abs() + 2.0 ** -25).all()
