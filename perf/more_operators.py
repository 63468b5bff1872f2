"""An 8-bit cache, its pages and beam search over it, as a serving program calls them.

Five kinds of pass:

``attend8``  attention of new tokens over a paged cache of e4m3 codes with a
             power-of-two scale for each block of tokens and head.
``append8``  new tokens' keys and values into such a cache, rotated on the way,
             and the values that their blocks then hold.
``fork``     sequences take over other sequences' pages (samples of a prompt,
             beams): tables and counts, the last pages copied, room for the
             next token.
``churn``    some sequences end, the pool is compacted, others get pages.
``beam``     the best continuations over beams and vocabulary, and the beams'
             token histories in their new order.

``own`` chooses between the plain form (torch, 32 bits; 64 for angles and the
scores of a beam search) and the entry points of ``paper_2605_05819_amd.cl``.
"""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
E4M3 = torch.float8_e4m3fn
# the scales' exponents that keep every value finite and normal in the cache's type (fp16: whole in its subnormals)
EXPONENTS = {"fp16": (-15, 8), "bf16": (-117, 120)}


# ------------------------------------------------------------------- the cases

def listed():
    return [
        # Single-stream decoding in the Llama-3.1-8B layer's shape (4096 / 1024
        # projections): one token, a few thousand cached.
        _attend(name="attend8-T1", seqs=1, q_lo=1, q_hi=1, kv_lo=2049, kv_hi=2049, act="fp16", page=16, block=16),
        # An ordinary serving batch: conversations of one token to 8192.
        _attend(name="attend8-T16-ragged", seqs=16, q_lo=1, q_hi=1, kv_lo=1, kv_hi=8192, act="bf16", page=64, block=16),
        # Four long documents, four drafted tokens each: the largest read.
        _attend(name="attend8-T4x4-long", seqs=4, q_lo=4, q_hi=4, kv_lo=100003, kv_hi=131072, act="fp16", page=64,
                block=64),
        # 64 beams behind one prompt of 8192 tokens.
        _attend(name="attend8-prefix-T64", seqs=64, q_lo=1, q_hi=1, kv_lo=17, kv_hi=777, act="bf16", page=32, block=32,
                prefix=8192),
        # Prompts of odd lengths behind cached turns, the longest 7001 of 9001: the largest product.
        _attend(name="attend8-prompts-ragged", seqs=4, q_lo=700, q_hi=7001, kv_lo=1400, kv_hi=9001, act="bf16",
                page=16, block=16),
        # A decode step of 64 sequences, most of them in the middle of a block.
        _append(name="append8-T64", seqs=64, q_lo=1, q_hi=1, kv_lo=5, kv_hi=8192, act="fp16", page=16, block=16),
        # Ragged prompts, 8 k tokens in all, with per-head norms.
        _append(name="append8-prompts", seqs=7, q_lo=100, q_hi=4001, kv_lo=100, kv_hi=30000, act="bf16", page=64,
                block=32, norm=True, interleaved=True, rot=64),
        # Four samples of one prompt: the smallest call.
        _fork(name="fork-samples", groups=1, beams=4, kv_lo=300, kv_hi=300, act="fp16", page=16, layers=2, fresh=True),
        # A beam step of 16 requests: eight layers' caches of 4 beams each.
        _fork(name="fork-beams", groups=16, beams=4, kv_lo=500, kv_hi=2000, act="bf16", page=32, layers=8),
        # Half of 32 requests end, the pool is compacted, as many are admitted.
        _churn(name="churn-32", seqs=32, kv_lo=100, kv_hi=4000, act="bf16", page=64, layers=4),
        # One request's beams over a small vocabulary.
        _beam(name="beam-1x4", groups=1, beams=4, vocab=32000, act="fp32", length=100),
        # 16 requests of 8 beams over a large one, hypotheses of several lengths, some of them finished.
        _beam(name="beam-16x8", groups=16, beams=8, vocab=128000, act="bf16", alpha=0.6, finished=0.2, length=1000),
    ]


def _named(c, name):
    return dict(c, name=name) if name else c


def _attend(name=None, seqs=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, act="fp16", page=16, block=16, q_heads=32, kv_heads=8,
            dim=128, prefix=0, window=0, causal=True):
    return _named({"op": "attend8", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi,
                   "act": act, "page": page, "block": block, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
                   "prefix": prefix, "window": window, "causal": causal}, name)


def _append(name=None, seqs=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, act="fp16", page=16, block=16, q_heads=32, kv_heads=8,
            dim=128, rot=128, interleaved=False, norm=False):
    return _named({"op": "append8", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi,
                   "act": act, "page": page, "block": block, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
                   "prefix": 0, "rot": rot, "interleaved": interleaved, "norm": norm}, name)


def _fork(name=None, groups=1, beams=4, kv_lo=1, kv_hi=1, act="fp16", page=16, kv_heads=8, dim=128, layers=2, fresh=False):
    return _named({"op": "fork", "groups": groups, "beams": beams, "kv_lo": kv_lo, "kv_hi": kv_hi, "act": act,
                   "page": page, "kv_heads": kv_heads, "dim": dim, "layers": layers, "fresh": fresh}, name)


def _churn(name=None, seqs=2, kv_lo=1, kv_hi=1, act="fp16", page=16, kv_heads=8, dim=128, layers=2):
    return _named({"op": "churn", "seqs": seqs, "kv_lo": kv_lo, "kv_hi": kv_hi, "act": act, "page": page,
                   "kv_heads": kv_heads, "dim": dim, "layers": layers}, name)


def _beam(name=None, groups=1, beams=4, picks=0, vocab=32000, act="fp32", alpha=0.0, finished=0.0, length=100):
    return _named({"op": "beam", "groups": groups, "beams": beams, "picks": picks or beams, "vocab": vocab, "act": act,
                   "alpha": alpha, "finished": finished, "length": length}, name)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attend8", "attend8", "attend8", "append8", "fork", "churn", "beam", "beam"))
    act = rng.choice(("fp16", "bf16"))
    kv_heads, group = rng.choice(((8, 4), (8, 4), (4, 8), (2, 7), (8, 1), (1, 16)))
    dim = rng.choice((128, 128, 64, 256))
    page = rng.choice((16, 32, 64, 128))
    block = min(page, rng.choice((1, 8, 16, 16, 32, 64)))
    heads = {"q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "act": act, "page": page, "block": block}
    if op == "attend8":
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
    if op == "append8":
        q_hi = rng.choice((1, _log(rng, 2, 4096)))
        return _append(seqs=_log(rng, 1, 64) if q_hi == 1 else rng.randint(1, 6), q_lo=_log(rng, 1, q_hi), q_hi=q_hi,
                       kv_lo=q_hi, kv_hi=_log(rng, q_hi, 40000), rot=dim // rng.choice((1, 1, 2)),
                       interleaved=rng.random() < 0.5, norm=rng.random() < 0.5, **heads)
    pool = {"kv_heads": kv_heads, "dim": dim, "act": act, "page": page}
    if op == "fork":
        kv_hi = _log(rng, 10, 3000)
        return _fork(groups=_log(rng, 1, 24), beams=rng.randint(2, 8), kv_lo=_log(rng, 1, kv_hi), kv_hi=kv_hi,
                     layers=rng.randint(1, 4), fresh=rng.random() < 0.3, **pool)
    if op == "churn":
        kv_hi = _log(rng, 50, 4000)
        return _churn(seqs=_log(rng, 2, 32), kv_lo=_log(rng, 1, kv_hi), kv_hi=kv_hi, layers=rng.randint(1, 3), **pool)
    beams = rng.randint(1, 12)
    vocab = _log(rng, 300, 150000)
    return _beam(groups=_log(rng, 1, max(1, min(64, 16_000_000 // (vocab * beams)))), beams=beams,
                 picks=beams * rng.choice((1, 1, 2)), vocab=vocab, act=rng.choice(("fp32", act)),
                 alpha=rng.choice((0.0, 0.6, 1.0)), finished=rng.choice((0.0, 0.3)), length=_log(rng, 1, 2000))


def _spread(lo, hi, n):
    return [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) if n > 1 else hi for i in range(n)]


def _lengths(case):
    """The sequences' new tokens and keys of their own: spread over the logarithm of their ranges, no
    sequence with fewer keys than new tokens."""
    n = case["seqs"]
    q = _spread(case["q_lo"], case["q_hi"], n)
    own_kv = _spread(case["kv_lo"], case["kv_hi"], n)
    return q, [max(a, b) for a, b in zip(q, own_kv)]


def _parents(case):
    """Which beam of its request each beam continues: some twice, some not at all."""
    rng = random.Random(100 * case["groups"] + case["beams"])
    n = case["beams"]
    if case["fresh"]:                     # every sample from the one sequence of its request
        return [g * n for g in range(case["groups"]) for _ in range(n)]
    return [g * n + rng.randrange(n) for g in range(case["groups"]) for _ in range(n)]


def work(case):
    c = case
    if c["op"] == "attend8":
        q, kv = _lengths(case)
        P, S = c["prefix"], c["page"]
        pairs, read = 0, 0
        for a, n in zip(q, kv):
            n += P
            first = n                       # lowest key that one of the new tokens sees
            for i in range(a):
                p = n - a + i if c["causal"] else n - 1
                lo = max(0, (n - a + i) - c["window"] + 1) if c["window"] else 0
                pairs += max(0, p + 1 - lo)
                first = min(first, lo)
            read += n - max(first, P)
        width = 2 * c["kv_heads"] * (c["dim"] + 1.0 / c["block"])    # a key's and its value's bytes, their scales
        bytes_ = int((read + P) * width) + 4 * sum(q) * c["q_heads"] * c["dim"] + 4 * sum(-(-n // S) for n in kv)
        return {"bytes": bytes_, "flops": 4 * pairs * c["q_heads"] * c["dim"]}
    if c["op"] == "append8":
        q, kv = _lengths(case)
        held = sum(a + (n - a) % c["block"] for a, n in zip(q, kv))
        tokens, row = sum(q), c["kv_heads"] * c["dim"]
        return {"bytes": 4 * tokens * c["q_heads"] * c["dim"] + 6 * tokens * row + 6 * held * row,
                "flops": 6 * tokens * (c["q_heads"] + 2 * c["kv_heads"]) * c["dim"]}
    if c["op"] == "fork":
        kv = [n for n in _spread(c["kv_lo"], c["kv_hi"], c["groups"]) for _ in range(c["beams"])]
        at = _parents(case)
        copies = sum(kv[p] % c["page"] != 0 and p in at[:i] for i, p in enumerate(at))
        page = 2 * c["kv_heads"] * c["page"] * c["dim"]
        return {"bytes": 2 * copies * page * 2 * c["layers"] + 8 * sum(-(-n // c["page"]) for n in kv), "flops": 0}
    if c["op"] == "churn":
        pages = [-(-n // c["page"]) for n in _spread(c["kv_lo"], c["kv_hi"], c["seqs"])]
        moved = min(sum(pages[0::2]), sum(pages[1::2]))
        page = 2 * c["kv_heads"] * c["page"] * c["dim"]
        return {"bytes": 2 * moved * page * 2 * c["layers"] + 8 * sum(pages), "flops": 0}
    rows = c["groups"] * c["beams"]
    size = 4 if c["act"] == "fp32" else 2
    alive = rows - int(c["finished"] * c["beams"]) * c["groups"]
    return {"bytes": alive * c["vocab"] * size + 4 * (rows + c["groups"] * c["picks"]) * c["length"] + 32 * rows,
            "flops": 4 * alive * c["vocab"]}


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
    s = SimpleNamespace(case=case, q=q, kv=[n + P for n in kv], num_pages=pool.numel(), table=table,
                        prefix=pool[:shared].contiguous() if P else None)
    s.q_len, s.kv_len = _int32(q), _int32(s.kv)
    s.start, s.tokens = _starts(q), sum(q)
    s.max_q, s.max_kv = max(q), max(s.kv)
    return s


def _starts(q):
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    return _int32(start)


def _codes(gen, case, s):
    """Codes and scales as appends leave them: values of unit size and more, each block's by its own exponent."""
    shape = (s.num_pages, case["kv_heads"], case["page"], case["dim"])
    codes = _normal(gen, shape, torch.float32, 64.0).clamp_(-448.0, 448.0).to(E4M3).view(torch.uint8)
    scales = torch.randint(120, 123, shape[:2] + (case["page"] // case["block"],), generator=gen, device=DEV,
                           dtype=torch.int32).to(torch.uint8)
    return codes, scales


def _handles(s):
    """The cache and batch descriptors a serving program keeps beside its buffers."""
    from paper_2605_05819_amd import cl
    s.cache = cl.KvCache8(s.k, s.v, s.k_scale, s.v_scale, DTYPES[s.case["act"]])
    even = min(s.q) == max(s.q)
    s.batch = cl.KvBatch(s.kv_len, s.table, s.tokens, q_len=s.max_q, q_start=None if even else s.start,
                         max_kv_len=s.max_kv, prefix_table=s.prefix, prefix_len=s.case["prefix"])
    return cl


def _prepare_cache(case, seed, gen):
    act = DTYPES[case["act"]]
    s = _batch(case, seed, gen)
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["dim"]
    s.k, s.k_scale = _codes(gen, case, s)
    s.v, s.v_scale = _codes(gen, case, s)
    if case["op"] == "attend8":
        # heads from diffuse to sharp
        sharp = torch.linspace(0.5, 3.0, Hq, device=DEV)[:, None]
        s.qx = (_normal(gen, (s.tokens, Hq, D), torch.float32) * sharp).to(act)
        s.out = torch.empty((s.tokens, Hq, D), dtype=act, device=DEV)
        if own:
            cl = _handles(s)
            s.ws = cl.workspace(cl.attention_workspace(s.cache, s.batch, Hq), DEV)
        return s
    s.qx = _normal(gen, (s.tokens, Hq, D), act)
    s.kx = _normal(gen, (s.tokens, Hkv, D), act, 2.0)
    s.vx = _normal(gen, (s.tokens, Hkv, D), act)
    # the frequencies of a base of 500000, as a model's configuration gives them
    j = torch.arange(case["rot"] // 2, dtype=torch.float64)
    s.freq = (500000.0 ** (-2.0 * j / case["rot"])).to(torch.float32).to(DEV)
    s.qw = 1 + _normal(gen, (D,), torch.float32, 0.1).to(act) if case["norm"] else None
    s.kw = 1 + _normal(gen, (D,), torch.float32, 0.1).to(act) if case["norm"] else None
    s.out = torch.empty_like(s.qx)
    # what is read back: every sequence's blocks that the new tokens reach, from their first row on
    s.held = [a + (n - a) % case["block"] for a, n in zip(s.q, s.kv)]
    s.held_len, s.held_start, s.rows = _int32(s.held), _starts(s.held), sum(s.held)
    s.k_held = torch.empty((s.rows, Hkv, D), dtype=act, device=DEV)
    s.v_held = torch.empty_like(s.k_held)
    if own:
        cl = _handles(s)
        s.rope = cl.Rope(s.freq, interleaved=case["interleaved"])
        s.reading = cl.KvBatch(s.kv_len, s.table, s.rows, q_len=max(s.held), q_start=s.held_start, max_kv_len=s.max_kv)
    return s


def _prepare_pages(case, seed, gen):
    """Tables over a pool with a count of holders for each page; pages scattered, some of them free."""
    S, n = case["page"], case.get("beams", 1)
    lens = _spread(case["kv_lo"], case["kv_hi"], case["groups"] if case["op"] == "fork" else case["seqs"])
    lens = [x for x in lens for _ in range(n)]
    width = max(lens) // S + 1
    rows, taken = [], 0
    for i, x in enumerate(lens):
        full, used = x // S, -(-x // S)
        if case["op"] == "fork" and case["fresh"] and i % n:
            rows.append([])               # a row without a sequence
            lens[i] = 0
        elif case["op"] == "fork" and i % n:
            rows.append(rows[i - i % n][:full] + list(range(taken, taken + used - full)))
            taken += used - full
        else:
            rows.append(list(range(taken, taken + used)))
            taken += used
    s = SimpleNamespace(case=case, num_pages=taken + 2 * len(lens) + 5, turn=0)
    names = torch.randperm(s.num_pages, generator=gen, device=DEV).to(torch.int32)
    flat = torch.full((len(rows), width), -1, dtype=torch.int64)
    for i, r in enumerate(rows):
        flat[i, :len(r)] = torch.tensor(r, dtype=torch.int64)
    flat = flat.to(DEV)
    s.table = torch.where(flat >= 0, names[flat.clamp(min=0)], -1)
    s.kv_len = _int32(lens)
    s.refs = torch.bincount(s.table[s.table >= 0].long(), minlength=s.num_pages).to(torch.int32)
    s.pool = _normal(gen, (2 * case["layers"], s.num_pages, case["kv_heads"], S, case["dim"]), DTYPES[case["act"]])
    if case["op"] == "fork":
        s.parents = _int32(_parents(case))
        s.table2, s.kv_len2 = torch.empty_like(s.table), torch.empty_like(s.kv_len)
    else:
        # every second sequence, then the others
        even = torch.arange(len(lens), dtype=torch.int32, device=DEV)
        s.rows = (even[0::2].contiguous(), even[1::2].contiguous())
        s.want = s.kv_len.clone()
    if own:
        from paper_2605_05819_amd import cl
        s.pages = cl.PagePool(s.refs, S, [cl.KvCache(k, v) for k, v in zip(s.pool[0::2], s.pool[1::2])])
    return s


def _prepare_beam(case, seed, gen):
    s = SimpleNamespace(case=case)
    G, n, V = case["groups"], case["beams"], case["vocab"]
    rows = G * n
    s.logits = _normal(gen, (rows, V), DTYPES[case["act"]], 2.0)
    s.eos = V // 2
    s.length = torch.randint(1, case["length"] + 1, (rows,), generator=gen, device=DEV, dtype=torch.int32)
    s.scores = -3.0 * torch.rand((rows,), generator=gen, device=DEV) * s.length.float().sqrt()
    s.done = (torch.arange(rows, device=DEV) % n < int(case["finished"] * n)).to(torch.int32)
    s.history = torch.randint(0, V, (rows, case["length"]), generator=gen, device=DEV, dtype=torch.int32)
    picks = G * case["picks"]
    s.history2 = torch.empty((picks, case["length"]), dtype=torch.int32, device=DEV)
    if own:
        from paper_2605_05819_amd import cl
        s.rule = cl.Beams(n, picks=case["picks"], eos=s.eos, alpha=case["alpha"])
        s.ws = cl.workspace(cl.beam_workspace(s.rule, G, V), DEV)
    return s


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] in ("attend8", "append8"):
        return _prepare_cache(case, seed, gen)
    return _prepare_beam(case, seed, gen) if case["op"] == "beam" else _prepare_pages(case, seed, gen)


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
    k, v = cl.kv_read(s.cache, s.reading, k=s.k_held, v=s.v_held)
    return q, k, v


def _own_fork(s):
    from paper_2605_05819_amd import cl
    cl.kv_fork(s.pages, s.table, s.kv_len, s.parents, room=1, table_out=s.table2, kv_len_out=s.kv_len2)
    return _forked(s)


def _forked(s):
    """The new tables take the old ones' place for the next step."""
    s.table, s.table2, s.kv_len, s.kv_len2 = s.table2, s.table, s.kv_len2, s.kv_len
    return s.table, s.kv_len, s.refs, s.pool


def _own_churn(s):
    from paper_2605_05819_amd import cl
    cl.kv_free(s.pages, s.table, s.kv_len, rows=s.rows[s.turn])
    cl.kv_compact(s.pages, [s.table])
    cl.kv_reserve(s.pages, s.table, s.kv_len, s.want)
    s.turn ^= 1
    return s.table, s.kv_len, s.refs, s.pool


def _own_beam(s):
    from paper_2605_05819_amd import cl
    scores, tokens, parents, length, done = cl.beam_select(s.rule, s.logits, s.scores, s.length, s.done, ws=s.ws)
    cl.gather_rows([s.history], parents, [s.history2])
    return scores, tokens, parents, length, done, s.history2


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


def _power(e):
    return torch.ldexp(torch.ones((), device=DEV), e)


def _values(s, codes, scales, page, row):
    """float32 [...][heads][dim] of the cache's rows."""
    e = scales[page, :, row // s.case["block"]].int() - 127
    return codes[page, :, row].view(E4M3).float() * _power(e)[..., None]


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
    k = _values(s, s.k, s.k_scale, page, row).permute(0, 2, 3, 1).contiguous()      # [B][Hkv][D][keys]
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
    v = _values(s, s.v, s.v_scale, page, row).permute(0, 2, 1, 3).contiguous()      # [B][Hkv][keys][D]
    o = torch.matmul(p.view(B, Hkv, g * s.max_q, s.max_kv), v).view(B, Hkv, g, s.max_q, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(B, s.max_q, Hq, D)[seq, place].to(s.qx.dtype)


def _exponent(most, lo, hi):
    """The smallest e with most <= 448 2^e, within lo..hi."""
    m, e = torch.frexp(most)
    return (torch.where(most > 0, e - 9 + (m > 0.875), lo)).clamp(lo, hi).int()


def _plain_append(s):
    c = s.case
    S, block, act = c["page"], c["block"], s.qx.dtype
    seq, place, pos = _positions(s)
    angle = pos.double()[:, None] * s.freq.double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

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
        return torch.cat((head, rest), -1)

    page, row = _rows(s, seq, pos)
    lo, hi = EXPONENTS[c["act"]]
    blocks = S // block
    at = page * blocks + row // block                                   # the token's block in the pool
    opens = (row % block == 0) | (place == 0)                           # first of its block among the new ones
    head_page, head_row = page[opens], row[opens]
    old = torch.arange(block, device=DEV)[None, :] < (head_row % block)[:, None]       # rows that stood there before

    def store(x, codes, scales):
        most = torch.zeros((s.num_pages * blocks, c["kv_heads"]), device=DEV)
        most.index_reduce_(0, at, x.abs().amax(-1), "amax")
        e = _exponent(most, lo, hi)
        e0 = scales[head_page, :, head_row // block].int() - 127
        e1 = torch.where(old.any(1, keepdim=True), torch.maximum(e[at[opens]], e0), e[at[opens]])
        e[at[opens]] = e1
        scales[head_page, :, head_row // block] = (e1 + 127).to(torch.uint8)
        rows = (head_row // block * block)[:, None] + torch.arange(block, device=DEV)[None, :]
        kept = codes[head_page[:, None], :, rows]                                       # [opens][block][heads][dim]
        less = (kept.view(E4M3).float() * _power(e0 - e1)[:, None, :, None]).to(E4M3).view(torch.uint8)
        codes[head_page[:, None], :, rows] = torch.where(old[:, :, None, None], less, kept)
        codes[page, :, row] = (x * _power(-e[at])[..., None]).to(E4M3).view(torch.uint8)

    store(turned(s.kx, s.kw), s.k, s.k_scale)
    store(s.vx.float(), s.v, s.v_scale)
    seq = torch.repeat_interleave(torch.arange(len(s.held), device=DEV), s.held_len.long(), output_size=s.rows)
    pos = s.kv_len.long()[seq] - s.held_len.long()[seq] + torch.arange(s.rows, device=DEV) - s.held_start.long()[seq]
    page, row = _rows(s, seq, pos)
    return (turned(s.qx, s.qw).to(act), _values(s, s.k, s.k_scale, page, row).to(act),
            _values(s, s.v, s.v_scale, page, row).to(act))


def _give_pages(s, table, asked):
    """The lowest free pages to the entries that ask, in order; -1 where there are none left."""
    free = (s.refs > 0).to(torch.int32).sort(stable=True).indices
    nth = asked.flatten().cumsum(0).view_as(table) - 1
    left = (s.refs == 0).sum()
    got = torch.where(nth < left, free[nth.clamp(0, s.num_pages - 1)], -1).to(torch.int32)
    table[asked] = got[asked]
    pages = table[asked]
    s.refs[pages[pages >= 0].long()] = 1


def _plain_fork(s):
    S, p = s.case["page"], s.parents.long()
    n, width = s.table.shape
    entry = torch.arange(width, device=DEV)[None, :]
    used = (s.kv_len + S - 1) // S
    children = torch.bincount(p, minlength=n)
    order = torch.arange(n, device=DEV)
    first = torch.full((n,), n, device=DEV).scatter_reduce_(0, p, order, "amin")[p] == order
    # holders: every child in place of the parent; pages kept ahead go to the first child
    more = torch.where(entry < used[:, None], children[:, None] - 1, torch.where(children > 0, 0, -1)[:, None])
    held = s.table >= 0
    s.refs.index_add_(0, s.table[held].long(), more[held].to(torch.int32))
    table = torch.where((entry < used[p][:, None]) | first[:, None], s.table[p], -1)
    s.kv_len2.copy_(s.kv_len[p])
    # a last page that another sequence holds too is copied; the next token's page
    last = entry == used[p][:, None] - 1
    page = torch.where(last, table, -1).amax(1)
    alone = first & (s.refs[page.clamp(min=0).long()] == children[p])
    copied = (s.kv_len2 % S != 0) & ~alone
    asked = (last & copied[:, None]) | ((entry >= used[p][:, None]) & (entry < ((s.kv_len2 + S) // S)[:, None]) & (table < 0))
    _give_pages(s, table, asked)
    new = torch.where(last, table, -1).amax(1)
    s.refs.index_add_(0, page[copied].long(), torch.full_like(page[copied], -1))
    there = copied & (new >= 0)
    s.pool[:, new[there].long()] = s.pool[:, page[there].long()]
    s.table2.copy_(table)
    return _forked(s)


def _plain_churn(s):
    S, rows = s.case["page"], s.rows[s.turn].long()
    s.turn ^= 1
    gone = s.table[rows]
    s.refs.index_add_(0, gone[gone >= 0].long(), torch.full_like(gone[gone >= 0], -1))
    s.table[rows] = -1
    s.kv_len[rows] = 0
    # the pages behind the first `live` ones move into the holes among those
    number = torch.arange(s.num_pages, device=DEV)
    live = (s.refs > 0).sum()
    movers = ((s.refs > 0) & (number >= live)).nonzero()[:, 0]
    holes = ((s.refs == 0) & (number < live)).nonzero()[:, 0]
    s.pool[:, holes] = s.pool[:, movers]
    s.refs[holes] = s.refs[movers]
    s.refs[movers] = 0
    number[movers] = holes
    s.table.copy_(torch.where(s.table >= 0, number[s.table.clamp(min=0).long()], -1))
    entry = torch.arange(s.table.shape[1], device=DEV)[None, :]
    _give_pages(s, s.table, (entry < ((s.want + S - 1) // S)[:, None]) & (s.table < 0))
    return s.table, s.kv_len, s.refs, s.pool


def _plain_beam(s):
    c = s.case
    G, n, V, k = c["groups"], c["beams"], c["vocab"], c["picks"]
    x = s.logits.double()
    m = x.amax(1, keepdim=True)
    x = x - (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))
    done = s.done.bool()[:, None]
    token = torch.arange(V, device=DEV)[None, :]
    total = s.scores.double()[:, None] + torch.where(done, torch.where(token == s.eos, 0.0, -math.inf), x)
    length = s.length + 1 - s.done
    rank = total / length.double()[:, None] ** c["alpha"]
    best = rank.view(G, n * V).sort(dim=1, descending=True, stable=True).indices[:, :k]
    row = (best // V + n * torch.arange(G, device=DEV)[:, None]).flatten()
    token = (best % V).flatten()
    ended = s.done.bool()[row] | (token == s.eos)
    s.history2.copy_(s.history[row])
    shape = (G, k)
    return (total[row, token].float().view(shape), token.int().view(shape), row.int().view(shape),
            length[row].int().view(shape), ended.int().view(shape), s.history2)


_run_own = {"attend8": _own_attend, "append8": _own_append, "fork": _own_fork, "churn": _own_churn, "beam": _own_beam}
_run_plain = {"attend8": _plain_attend, "append8": _plain_append, "fork": _plain_fork, "churn": _plain_churn,
              "beam": _plain_beam}


# ------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    if case["op"] in ("fork", "churn"):        # copies and whole numbers
        return None
    s = prepare(case, seed)
    return {"attend8": _exact_attend, "append8": _exact_append, "beam": _exact_beam}[case["op"]](s)


def _decoded(codes):
    """e4m3 by its fields: 1.f 2^(x - 7), or 0.f 2^-6."""
    u = codes.int()
    x, f = (u >> 3) & 15, (u & 7).double()
    size = torch.where(x > 0, (8 + f) * 2.0 ** (x - 10).double(), f * 2.0 ** -9)
    return torch.where(u >= 128, -size, size)


def _nearest(x):
    """x at the nearest e4m3 value, ties to even; |x| <= 448."""
    step = 2.0 ** (torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _sequence(s, b, codes, scales, n):
    """The first n rows of sequence b, [heads][n][dim], page by page."""
    P, S, block = s.case["prefix"], s.case["page"], s.case["block"]

    def rows(pages, count):
        e = scales[pages].double() - 127.0
        x = _decoded(codes[pages]) * (2.0 ** e).repeat_interleave(block, 2)[..., None]
        return x.transpose(0, 1).flatten(1, 2)[:, :count]

    parts = [rows(s.prefix.long(), P)] if P else []
    return torch.cat(parts + [rows(s.table[b, :-(-(n - P) // S)].long(), n - P)], 1)


def _exact_attend(s):
    c = s.case
    Hkv, D = c["kv_heads"], c["dim"]
    out, at = [], 0
    for b, (a, n) in enumerate(zip(s.q, s.kv)):
        k, v = _sequence(s, b, s.k, s.k_scale, n), _sequence(s, b, s.v, s.v_scale, n)
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
    rot, D, block = c["rot"], c["dim"], c["block"]
    lo, hi = EXPONENTS[c["act"]]
    half = torch.arange(rot // 2, device=DEV)
    first, second = (2 * half, 2 * half + 1) if c["interleaved"] else (half, half + rot // 2)
    q, k, v = s.qx.double(), s.kx.double(), s.vx.double()
    if c["norm"]:
        q = q / torch.sqrt((q * q).sum(-1, keepdim=True) / D + 1e-6) * s.qw.double()
        k = k / torch.sqrt((k * k).sum(-1, keepdim=True) / D + 1e-6) * s.kw.double()
    keys, values, at = [], [], 0
    for b, (a, n, held) in enumerate(zip(s.q, s.kv, s.held)):
        where = torch.arange(n - a, n, device=DEV)
        z = torch.polar(torch.ones((a, rot // 2), dtype=torch.float64, device=DEV),
                        where.double()[:, None] * s.freq.double())[:, None]
        for x in (q, k):
            part = x[at:at + a]
            turned = torch.complex(part[..., first], part[..., second]) * z
            part[..., first], part[..., second] = turned.real, turned.imag
        for new, codes, scales, to in ((k, s.k, s.k_scale, keys), (v, s.v, s.v_scale, values)):
            # whole blocks of rows: those from before, the new ones, nothing behind
            before = held - a
            x = torch.zeros((-(-held // block) * block, c["kv_heads"], D), dtype=torch.float64, device=DEV)
            x[before:held] = new[at:at + a]
            most = x.abs().amax(-1).view(-1, block, c["kv_heads"]).amax(1)      # [blocks][heads]
            e = torch.ceil(torch.log2((most / 448.0).clamp(min=2.0 ** lo))).clamp(lo, hi)
            if before:
                i = n - held
                page, row = s.table[b, i // c["page"]].long(), i % c["page"]
                e0 = scales[page, :, row // block].double() - 127.0
                e[0] = torch.maximum(e[0], e0)
                x[:before] = (_decoded(codes[page, :, row:row + before]) * (2.0 ** e0)[:, None, None]).transpose(0, 1)
            size = (2.0 ** e).repeat_interleave(block, 0)[..., None]
            to.append((_nearest(x / size) * size)[:held])
        at += a
    return q, torch.cat(keys), torch.cat(values)


def _exact_beam(s):
    c = s.case
    G, n, V, k = c["groups"], c["beams"], c["vocab"], c["picks"]
    picked = []
    for g in range(G):
        rows = slice(g * n, (g + 1) * n)
        over = s.done[rows].double()[:, None]
        each = torch.log_softmax(s.logits[rows].double(), 1) * (1 - over)
        each = each.masked_fill((over > 0) & (torch.arange(V, device=DEV) != s.eos), -math.inf)
        each = each + s.scores[rows].double()[:, None]
        rank = each / (s.length[rows].double()[:, None] + 1 - over) ** c["alpha"]
        picked.append(each.flatten()[torch.argsort(-rank.flatten(), stable=True)[:k]])
    return torch.stack(picked), None, None, None, None, None
