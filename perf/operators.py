"""The operators between a decoder layer's linears, as a serving program calls them.

Four kinds of pass:

``attend``  attention of new tokens over the paged cache of their sequences:
            single tokens, a few drafted tokens, ragged prompts, and a batch
            whose sequences share a long prefix.
``append``  new tokens' keys and values to the paged cache, rotated on the
            way, and the rotated queries.
``norm``    a block's output (an MoE layer's slots weighted and summed) into
            the residual stream, and the next block's normalised input.
``route``   router logits to expert ids, weights and per-slot ranks.

``own`` chooses between the plain form (torch, 32 bits) and the entry points of
``paper_2605_05819_amd.cl``.
"""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------- the cases

def listed():
    return [
        # Single-stream decoding in the Llama-3.1-8B layer's shape (4096 / 1024
        # projections): one token, a few thousand cached.
        _attend(name="attend-T1", seqs=1, q_lo=1, q_hi=1, kv_lo=2049, kv_hi=2049, act="fp16", page=16),
        # An ordinary serving batch: conversations of one token to 8192.
        _attend(name="attend-T16-ragged", seqs=16, q_lo=1, q_hi=1, kv_lo=1, kv_hi=8192, act="bf16", page=64),
        # Four long documents, four drafted tokens each: the largest read.
        _attend(name="attend-T4x4-long", seqs=4, q_lo=4, q_hi=4, kv_lo=100003, kv_hi=131072, act="fp16", page=64),
        # 64 requests under one system prompt of 8192 tokens.
        _attend(name="attend-prefix-T64", seqs=64, q_lo=1, q_hi=1, kv_lo=17, kv_hi=777, act="bf16", page=32,
                prefix=8192),
        # A 2048-token prompt, causal: the prefill workload's tokens.
        _attend(name="attend-prompt-2048", seqs=1, q_lo=2048, q_hi=2048, kv_lo=2048, kv_hi=2048, act="fp16", page=64),
        # Prompts of odd lengths behind cached turns, the longest 7001 of 9001: the largest product.
        _attend(name="attend-prompts-ragged", seqs=4, q_lo=700, q_hi=7001, kv_lo=1400, kv_hi=9001, act="bf16",
                page=16),
        # One token's keys and values.
        _append(name="append-T1", seqs=1, q_lo=1, q_hi=1, kv_lo=4097, kv_hi=4097, act="fp16", page=16),
        # Ragged prompts, 8 k tokens in all, with per-head norms.
        _append(name="append-prompts", seqs=7, q_lo=100, q_hi=4001, kv_lo=100, kv_hi=30000, act="bf16", page=64,
                norm=True, interleaved=True, rot=64),
        # The MoE layer's largest decode batch: eight slots a token summed into the residual.
        _norm(name="norm-moe-T64", T=64, d=2048, slots=8, act="fp16", kind="rms"),
        # A prompt, with norms before and after the block and a gate.
        _norm(name="norm-prompt-2048", T=2048, d=4096, slots=0, act="bf16", kind="rms", post=True, gate="token",
              alpha=1.0, beta=0.5),
        # The same batch's routing: 128 experts, 8 of them a token, ranks for two windows.
        _route(name="route-T64", T=64, E=128, k=8, act="fp32", score="softmax", ranks=2),
        # A long prompt's routing in groups with a balance bias.
        _route(name="route-prompt-4099", T=4099, E=256, k=8, act="fp32", score="sigmoid", bias=True, groups=8,
               top_groups=4),
    ]


def _attend(name=None, seqs=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, act="fp16", page=16, q_heads=32, kv_heads=8, dim=128,
            prefix=0, window=0, causal=True):
    c = {"op": "attend", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi, "act": act,
         "page": page, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "prefix": prefix, "window": window,
         "causal": causal}
    return dict(c, name=name) if name else c


def _append(name=None, seqs=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, act="fp16", page=16, q_heads=32, kv_heads=8, dim=128,
            rot=128, interleaved=False, norm=False):
    c = {"op": "append", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi, "act": act,
         "page": page, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "prefix": 0, "rot": rot,
         "interleaved": interleaved, "norm": norm}
    return dict(c, name=name) if name else c


def _norm(name=None, T=1, d=4096, slots=0, act="fp16", kind="rms", post=False, gate="none", alpha=1.0, beta=1.0):
    c = {"op": "norm", "T": T, "d": d, "slots": slots, "act": act, "kind": kind, "post": post, "gate": gate,
         "alpha": alpha, "beta": beta}
    return dict(c, name=name) if name else c


def _route(name=None, T=1, E=128, k=8, act="fp32", score="softmax", bias=False, groups=1, top_groups=1,
           renormalize=True, ranks=0):
    c = {"op": "route", "T": T, "E": E, "k": k, "act": act, "score": score, "bias": bias, "groups": groups,
         "top_groups": top_groups, "renormalize": renormalize, "ranks": ranks}
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attend", "attend", "attend", "append", "norm", "route"))
    act = rng.choice(("fp16", "bf16"))
    kv_heads, group = rng.choice(((8, 4), (8, 4), (4, 8), (2, 7), (8, 1), (1, 16)))
    dim = rng.choice((128, 128, 64, 256))
    page = rng.choice((16, 32, 64, 128))
    heads = {"q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "act": act, "page": page}
    if op == "attend":
        shape = rng.choice(("tokens", "tokens", "prefix", "prompts", "prompts"))
        if shape == "prompts":
            seqs = rng.randint(1, 5)
            q_hi = _log(rng, 9, 2000)
            kv_hi = q_hi + _log(rng, 1, 2000)
            # as many pairs of tokens as the plain form has room for
            kv_hi = max(q_hi, min(kv_hi, 800_000_000 // (seqs * kv_heads * group * q_hi)))
            return _attend(seqs=seqs, q_lo=_log(rng, 1, q_hi), q_hi=q_hi, kv_lo=_log(rng, 1, kv_hi), kv_hi=kv_hi,
                           window=rng.choice((0, 0, _log(rng, 16, 2000))), causal=rng.random() < 0.8, **heads)
        seqs = _log(rng, 1, 64)
        q = rng.choice((1, 1, 1, rng.randint(2, 8)))
        room = max(64, min(131072, 1_800_000_000 // (4 * seqs * kv_heads * dim)))
        kv_hi = _log(rng, 16, room)
        prefix = _log(rng, 256, 16384) if shape == "prefix" else 0
        if prefix:
            kv_hi = min(kv_hi, 2000, max(64, room - prefix))
        return _attend(seqs=seqs, q_lo=q, q_hi=q, kv_lo=_log(rng, 1, kv_hi), kv_hi=kv_hi, prefix=prefix,
                       window=0 if prefix else rng.choice((0, 0, 0, _log(rng, 16, 4096))), **heads)
    if op == "append":
        q_hi = rng.choice((1, _log(rng, 2, 4096)))
        return _append(seqs=_log(rng, 1, 64) if q_hi == 1 else rng.randint(1, 6), q_lo=_log(rng, 1, q_hi), q_hi=q_hi,
                       kv_lo=q_hi, kv_hi=_log(rng, q_hi, 40000), rot=dim // rng.choice((1, 1, 2)),
                       interleaved=rng.random() < 0.5, norm=rng.random() < 0.5, **heads)
    if op == "norm":
        d = rng.choice((8 * _log(rng, 32, 1024), _log(rng, 64, 8192)))
        slots = rng.choice((0, 0, 2, 8))
        return _norm(T=min(_log(rng, 1, 4096), 16_000_000 // (d * max(1, slots))), d=d, slots=slots, act=act,
                     kind=rng.choice(("rms", "layer")), post=rng.random() < 0.5,
                     gate=rng.choice(("none", "channel", "token")), alpha=rng.choice((1.0, 0.7)),
                     beta=rng.choice((1.0, 0.5)))
    groups, top = rng.choice(((1, 1), (1, 1), (8, 4), (4, 2)))
    E = groups * _log(rng, 16, 512 // groups)
    score = rng.choice(("softmax", "sigmoid"))
    return _route(T=_log(rng, 1, 8192), E=E, k=rng.randint(1, 8), act=rng.choice(("fp32", act)), score=score,
                  bias=score == "sigmoid" and rng.random() < 0.5, groups=groups, top_groups=top,
                  renormalize=rng.random() < 0.8, ranks=rng.choice((0, 0, 1, 3)))


def _lengths(case):
    """The sequences' new tokens and keys of their own: spread over the logarithm of their ranges, no
    sequence with fewer keys than new tokens."""
    def spread(lo, hi, n):
        return [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) if n > 1 else hi for i in range(n)]

    n = case["seqs"]
    q = spread(case["q_lo"], case["q_hi"], n)
    own_kv = spread(case["kv_lo"], case["kv_hi"], n)
    return q, [max(a, b) for a, b in zip(q, own_kv)]


def work(case):
    if case["op"] == "attend":
        q, kv = _lengths(case)
        P, S = case["prefix"], case["page"]
        pairs, read = 0, 0
        for a, n in zip(q, kv):
            n += P
            first = n                       # lowest key that one of the new tokens sees
            for i in range(a):
                p = n - a + i if case["causal"] else n - 1
                lo = max(0, (n - a + i) - case["window"] + 1) if case["window"] else 0
                pairs += max(0, p + 1 - lo)
                first = min(first, lo)
            read += n - max(first, P)
        width = 2 * case["kv_heads"] * case["dim"]          # a key's or a value's bytes
        bytes_ = 2 * (read + P) * width + 4 * sum(q) * case["q_heads"] * case["dim"] + 4 * sum(-(-n // S) for n in kv)
        return {"bytes": bytes_, "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    if case["op"] == "append":
        n = sum(_lengths(case)[0]) * (case["q_heads"] + 2 * case["kv_heads"]) * case["dim"]
        return {"bytes": 4 * n, "flops": 6 * n}
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        rows = max(1, case["slots"]) + 3 + (case["gate"] == "token")
        return {"bytes": 2 * rows * T * d + 4 * T * case["slots"] + 2 * d * (1 + case["post"] + (case["gate"] == "channel")),
                "flops": T * d * (2 * max(1, case["slots"]) + 8)}
    size = 4 if case["act"] == "fp32" else 2
    return {"bytes": case["T"] * (size * case["E"] + 8 * case["k"] + 4 * case["k"] * case["ranks"]),
            "flops": 4 * case["T"] * case["E"]}


# ------------------------------------------------------------------ the inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(gen, shape, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _batch(case, seed, gen):
    """Sequences in a random order, their pages scattered over the pool as an allocator leaves them."""
    q, kv = _lengths(case)
    order = list(range(case["seqs"]))
    random.Random(seed).shuffle(order)
    q, kv = [q[i] for i in order], [kv[i] for i in order]
    S, P = case["page"], case["prefix"]
    pages = [-(-n // S) for n in kv]
    shared = -(-P // S)
    width = max(pages)
    pool = torch.randperm(sum(pages) + shared + 3, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((len(q), width), dtype=torch.int32, device=DEV)
    at = shared
    for b, n in enumerate(pages):
        table[b, :n] = pool[at:at + n]
        at += n
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    s = SimpleNamespace(case=case, q=q, kv=[n + P for n in kv], num_pages=pool.numel(), table=table, tokens=start[-1],
                        prefix=pool[:shared].contiguous() if P else None, start=_int32(start),
                        q_len=_int32(q), kv_len=_int32([n + P for n in kv]), uniform=min(q) == max(q))
    s.max_q, s.max_kv = max(q), max(s.kv)
    return s


def _handles(s):
    """The cache and batch descriptors a serving program keeps beside its buffers."""
    from paper_2605_05819_amd import cl
    s.cache = cl.KvCache(s.k, s.v)
    s.batch = cl.KvBatch(s.kv_len, s.table, s.tokens, q_len=s.max_q, q_start=None if s.uniform else s.start,
                         max_kv_len=s.max_kv, prefix_table=s.prefix, prefix_len=s.case["prefix"])
    return cl


def prepare(case, seed):
    gen = _generator(seed)
    act = DTYPES[case["act"]]
    if case["op"] in ("attend", "append"):
        s = _batch(case, seed, gen)
        Hq, Hkv, D, S = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
        s.k = _normal(gen, (s.num_pages, Hkv, S, D), act)
        s.v = _normal(gen, (s.num_pages, Hkv, S, D), act)
        if case["op"] == "attend":
            # heads from diffuse to sharp
            sharp = torch.linspace(0.5, 3.0, Hq, device=DEV)[:, None]
            s.qx = (_normal(gen, (s.tokens, Hq, D), torch.float32) * sharp).to(act)
            s.out = torch.empty((s.tokens, Hq, D), dtype=act, device=DEV)
            if own:
                cl = _handles(s)
                s.ws = cl.workspace(cl.attention_workspace(s.cache, s.batch, Hq), DEV)
            return s
        s.qx = _normal(gen, (s.tokens, Hq, D), act)
        s.kx = _normal(gen, (s.tokens, Hkv, D), act)
        s.vx = _normal(gen, (s.tokens, Hkv, D), act)
        # the frequencies of a base of 500000, as a model's configuration gives them
        j = torch.arange(case["rot"] // 2, dtype=torch.float64)
        s.freq = (500000.0 ** (-2.0 * j / case["rot"])).to(torch.float32).to(DEV)
        s.qw = 1 + _normal(gen, (D,), torch.float32, 0.1).to(act) if case["norm"] else None
        s.kw = 1 + _normal(gen, (D,), torch.float32, 0.1).to(act) if case["norm"] else None
        s.out = torch.empty_like(s.qx)
        if own:
            cl = _handles(s)
            s.rope = cl.Rope(s.freq, interleaved=case["interleaved"])
        return s
    if case["op"] == "norm":
        T, d, n = case["T"], case["d"], case["slots"]
        s = SimpleNamespace(case=case)
        s.y = _normal(gen, (T, n, d) if n else (T, d), act)
        s.slot_weights = torch.softmax(_normal(gen, (T, n), torch.float32), 1) if n else None
        s.res = _normal(gen, (T, d), act, 4.0)
        s.w = (1 + _normal(gen, (d,), torch.float32, 0.2)).to(act)
        s.post = (1 + _normal(gen, (d,), torch.float32, 0.2)).to(act) if case["post"] else None
        s.gate = {"none": None, "channel": (d,), "token": (T, d)}[case["gate"]]
        s.gate = _normal(gen, s.gate, act) if s.gate else None
        s.h = torch.empty((T, d), dtype=act, device=DEV)
        s.n = torch.empty((T, d), dtype=act, device=DEV)
        return s
    s = SimpleNamespace(case=case)
    T, E, k = case["T"], case["E"], case["k"]
    s.logits = _normal(gen, (T, E), act)
    # a balance bias moves in steps of a thousandth
    s.bias = torch.randint(-60, 61, (E,), generator=gen, device=DEV).float() * 0.001 if case["bias"] else None
    levels = _int32([0, 8, 16, 32])
    s.levels = (0, 8, 16, 32)
    s.ranks = [levels[torch.randint(0, 4, (E,), generator=gen, device=DEV)] for _ in range(case["ranks"])]
    s.ids = torch.empty((T, k), dtype=torch.int32, device=DEV)
    s.weights = torch.empty((T, k), dtype=torch.float32, device=DEV)
    s.slot_ranks = [torch.empty((T, k), dtype=torch.int32, device=DEV) for _ in range(case["ranks"])]
    if own:
        from paper_2605_05819_amd import cl
        s.router = cl.Router(E, k, score=case["score"], bias=s.bias, groups=case["groups"],
                             top_groups=case["top_groups"], group_best=2 if case["bias"] else 1,
                             renormalize=case["renormalize"])
    return s


# ------------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)[s.case["op"]](s)


def _own_attend(s):
    from paper_2605_05819_amd import cl
    return cl.attention(s.cache, s.batch, s.qx, window=s.case["window"], causal=s.case["causal"], out=s.out, ws=s.ws)


def _own_append(s):
    from paper_2605_05819_amd import cl
    q = cl.kv_append(s.cache, s.batch, s.kx, s.vx, q=s.qx, rope=s.rope, q_norm=s.qw, k_norm=s.kw, eps=1e-6,
                     q_out=s.out)
    return q, s.k, s.v


def _own_norm(s):
    from paper_2605_05819_amd import cl
    c = s.case
    return cl.residual_norm(s.y, s.w, residual=s.res, slot_weights=s.slot_weights, post_weight=s.post, gate=s.gate,
                            kind=c["kind"], eps=1e-6, alpha=c["alpha"], beta=c["beta"], h=s.h, out=s.n)


def _own_route(s):
    from paper_2605_05819_amd import cl
    if s.ranks:
        return cl.moe_route(s.router, s.logits, expert_ranks=s.ranks, levels=s.levels, ids=s.ids, weights=s.weights,
                            slot_ranks=s.slot_ranks)
    return cl.moe_route(s.router, s.logits, ids=s.ids, weights=s.weights)


# ------------------------------------------------------- the plain form, 32 bits

def _positions(s):
    """Sequence, place in it and position of every token."""
    seq = torch.repeat_interleave(torch.arange(len(s.q), device=DEV), s.q_len.long(), output_size=s.tokens)
    place = torch.arange(s.tokens, device=DEV) - s.start.long()[seq]
    return seq, place, s.kv_len.long()[seq] - s.q_len.long()[seq] + place


def _rows(s, seq, pos):
    """The page and the row in it of position ``pos`` of sequence ``seq``."""
    P, S = s.case["prefix"], s.case["page"]
    mine = (pos - P).clamp(0, s.table.shape[1] * S - 1)
    page = s.table[seq, mine // S].long()
    row = mine % S
    if P:
        both = pos.clamp(0, P - 1)
        shared = pos < P
        page = torch.where(shared, s.prefix[both // S].long(), page)
        row = torch.where(shared, both % S, row)
    return page, row


def _plain_attend(s):
    c = s.case
    B, Hq, Hkv, D, P = len(s.q), c["q_heads"], c["kv_heads"], c["dim"], c["prefix"]
    g = Hq // Hkv
    seq, place, pos = _positions(s)
    q = torch.zeros((B, s.max_q, Hq, D), device=DEV)
    q[seq, place] = s.qx.float() * (1.0 / math.sqrt(D))
    q = q.view(B, s.max_q, Hkv, g, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * s.max_q, D)
    key = torch.arange(s.max_kv, device=DEV)
    page, row = _rows(s, torch.arange(B, device=DEV)[:, None], key[None, :])
    k = s.k[page, :, row].float().permute(0, 2, 3, 1).contiguous()             # [B][Hkv][D][keys]
    score = torch.matmul(q, k).view(B, Hkv, g, s.max_q, s.max_kv)
    del k
    at = (s.kv_len.long() - s.q_len.long())[:, None] + torch.arange(s.max_q, device=DEV)[None, :]
    seen = (key < s.kv_len[:, None])[:, None, :]
    if c["causal"]:
        seen = seen & (key <= at[:, :, None])
    if c["window"]:
        seen = seen & (key > at[:, :, None] - c["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    m = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    v = s.v[page, :, row].float().permute(0, 2, 1, 3).contiguous()             # [B][Hkv][keys][D]
    o = torch.matmul(p.view(B, Hkv, g * s.max_q, s.max_kv), v).view(B, Hkv, g, s.max_q, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(B, s.max_q, Hq, D)[seq, place].to(s.qx.dtype)


def _plain_append(s):
    c = s.case
    seq, _, pos = _positions(s)
    angle = pos.float()[:, None] * s.freq
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        head, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["interleaved"]:
            a, b = head[..., 0::2], head[..., 1::2]
            head = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        else:
            a, b = head.chunk(2, -1)
            head = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
        return torch.cat((head, rest), -1).to(s.qx.dtype)

    page, row = _rows(s, seq, pos)
    s.k[page, :, row] = turned(s.kx, s.kw)
    s.v[page, :, row] = s.vx
    return turned(s.qx, s.qw), s.k, s.v


def _plain_norm(s):
    c = s.case

    def normed(x):
        if c["kind"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    u = (s.y.float() * s.slot_weights[..., None]).sum(1) if c["slots"] else s.y.float()
    if s.post is not None:
        u = normed(u) * s.post.float()
    if s.gate is not None:
        u = u * s.gate.float()
    h = c["alpha"] * s.res.float() + c["beta"] * u
    return h.to(s.res.dtype), (normed(h) * s.w.float()).to(s.res.dtype)


def _plain_route(s):
    c = s.case
    T, E, k = c["T"], c["E"], c["k"]
    x = s.logits.float()
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-x))
    # both scores rise with the logit: without a bias the logits decide, ties between equal ones only
    choice = p + s.bias if c["bias"] else x
    if c["groups"] > 1:
        best = choice.view(T, c["groups"], -1).sort(dim=-1, descending=True).values[..., :2 if c["bias"] else 1].sum(-1)
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        open_ = torch.zeros((T, c["groups"]), dtype=torch.bool, device=DEV).scatter_(1, kept, True)
        choice = choice.masked_fill(~open_.repeat_interleave(E // c["groups"], 1), -math.inf)
    ids = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, ids)
    if c["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    if not s.ranks:
        return ids.int(), w
    levels = torch.tensor(s.levels, device=DEV)
    # the nearest level to k w r, ties to the lower one
    near = [(levels - (k * w * r[ids].float())[..., None]).abs().argmin(-1) for r in s.ranks]
    return ids.int(), w, [levels[n].int() for n in near]


_run_own = {"attend": _own_attend, "append": _own_append, "norm": _own_norm, "route": _own_route}
_run_plain = {"attend": _plain_attend, "append": _plain_append, "norm": _plain_norm, "route": _plain_route}


# ------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "norm": _exact_norm, "route": _exact_route}[case["op"]](s)


def _sequence(s, b, pool, n):
    """The first n rows of sequence b, [heads][n][dim], gathered page by page."""
    P, S = s.case["prefix"], s.case["page"]
    parts = []
    if P:
        parts.append(pool[s.prefix.long()].transpose(0, 1).flatten(1, 2)[:, :P])
    mine = s.table[b, :-(-(n - P) // S)].long()
    parts.append(pool[mine].transpose(0, 1).flatten(1, 2)[:, :n - P])
    return torch.cat(parts, 1).double()


def _exact_attend(s):
    c = s.case
    Hkv, D = c["kv_heads"], c["dim"]
    out, at = [], 0
    for b, (a, n) in enumerate(zip(s.q, s.kv)):
        k, v = _sequence(s, b, s.k, n), _sequence(s, b, s.v, n)
        q = s.qx[at:at + a].double()                                            # [a][Hq][D]
        at += a
        i = torch.arange(n - a, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None, :]
        hidden = torch.zeros((a, n), dtype=torch.bool, device=DEV)
        if c["causal"]:
            hidden |= j > i
        if c["window"]:
            hidden |= j <= i - c["window"]
        heads = []
        for h in range(c["q_heads"]):
            x = (q[:, h] @ k[h * Hkv // c["q_heads"]].t().contiguous()) / D ** 0.5
            x[hidden] = -math.inf
            p = torch.exp(x - x.max(1, keepdim=True).values)
            heads.append((p @ v[h * Hkv // c["q_heads"]]) / p.sum(1, keepdim=True))
        out.append(torch.stack(heads, 1))
    return torch.cat(out)


def _exact_append(s):
    c = s.case
    rot, D = c["rot"], c["dim"]
    lo = torch.arange(rot // 2, device=DEV)
    first, second = (2 * lo, 2 * lo + 1) if c["interleaved"] else (lo, lo + rot // 2)
    q, k, v = s.qx.double(), s.kx.double(), s.vx.double()
    if c["norm"]:
        q = q / torch.sqrt((q * q).sum(-1, keepdim=True) / D + 1e-6) * s.qw.double()
        k = k / torch.sqrt((k * k).sum(-1, keepdim=True) / D + 1e-6) * s.kw.double()
    keys, values = s.k.double(), s.v.double()
    qs, at = [], 0
    for b, (a, n) in enumerate(zip(s.q, s.kv)):
        where = torch.arange(n - a, n, device=DEV)
        z = torch.polar(torch.ones((a, rot // 2), dtype=torch.float64, device=DEV),
                        where.double()[:, None] * s.freq.double())[:, None]
        for x in (q, k):
            part = x[at:at + a]
            turned = torch.complex(part[..., first], part[..., second]) * z
            part[..., first], part[..., second] = turned.real, turned.imag
        page = s.table[b].long()[where // c["page"]]
        keys[page, :, where % c["page"]] = k[at:at + a]
        values[page, :, where % c["page"]] = v[at:at + a]
        at += a
    return q, keys, values


def _exact_norm(s):
    c = s.case

    def statistics(x):
        mean = x.sum(1, keepdim=True) / c["d"] if c["kind"] == "layer" else 0.0
        return (x - mean) / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / c["d"] + 1e-6)

    u = s.y.double()
    if c["slots"]:
        u = torch.bmm(s.slot_weights.double()[:, None], u)[:, 0]
    if c["post"]:
        u = statistics(u) * s.post.double()
    if c["gate"] != "none":
        u = u * s.gate.double()
    h = c["alpha"] * s.res.double() + c["beta"] * u
    return h, statistics(h) * s.w.double()


def _exact_route(s):
    c = s.case
    x = s.logits.double()
    p = torch.softmax(x, 1) if c["score"] == "softmax" else torch.sigmoid(x)
    choice = p + s.bias.double() if c["bias"] else x
    T, E, G = c["T"], c["E"], c["groups"]
    if G > 1:
        by = torch.topk(choice.view(T, G, E // G), 2 if c["bias"] else 1, -1).values.sum(-1)
        place = torch.argsort(torch.argsort(-by, dim=1, stable=True), dim=1)
        choice = torch.where((place < c["top_groups"]).repeat_interleave(E // G, 1), choice, -math.inf)
    w = p.gather(1, torch.argsort(-choice, dim=1, stable=True)[:, :c["k"]])
    if c["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    return (None, w, [None] * len(s.ranks)) if s.ranks else (None, w)
