"""cl_kv_append, cl_moe_route and cl_residual_norm against the fp64 oracle, and a
decoder layer's step that runs them together with cl_attention."""

import math

import numpy as np
import pytest
import torch

from oracle import layer
from paper_2605_05819_amd import cl, workloads as wl
from tests.helpers import UNIT_ROUNDOFF, out_to_numpy

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def i32(a):
    return torch.tensor(np.asarray(a, np.int32)).cuda()


def rnd(g, shape, dtype, std=1.0):
    return torch.from_numpy((g.standard_normal(shape) * std).astype(np.float32)).to(dtype)


# --------------------------------------------------------------------- append

def _append_case(q_lens, kv_lens, Hq, Hkv, D, page, dtype, prefix=0, seed=0):
    g = np.random.default_rng(seed)
    B, N = len(q_lens), sum(q_lens)
    need = [-(-max(0, n - prefix) // page) for n in kv_lens]
    total = sum(need) + 2
    pool = g.permutation(total).astype(np.int32)
    table, at = np.full((B, max(need + [1])), -1, np.int32), 0
    for b in range(B):
        table[b, :need[b]] = pool[at:at + need[b]]
        at += need[b]
    kv0 = [rnd(g, (total, Hkv, page, D), dtype) for _ in range(2)]
    cache = cl.KvCache(kv0[0].cuda(), kv0[1].cuda())
    batch = cl.KvBatch(i32(kv_lens), i32(table), N, q_len=max(q_lens), q_start=i32(np.concatenate([[0], np.cumsum(q_lens)])),
                       max_kv_len=max(kv_lens), prefix_table=i32([0] * -(-prefix // page)) if prefix else None,
                       prefix_len=prefix)
    q, k, v = rnd(g, (N, Hq, D), dtype), rnd(g, (N, Hkv, D), dtype), rnd(g, (N, Hkv, D), dtype)
    return cache, batch, table, kv0, q, k, v


APPENDS = [
    # q_lens, kv_lens, Hq, Hkv, D, page, rot, interleaved, norm, prefix
    ([1], [1], 4, 2, 128, 16, 128, False, False, 0),
    ([1, 1, 1], [4097, 17, 130000], 32, 8, 128, 64, 128, False, True, 0),
    ([5, 1, 300], [5, 64, 1000], 7, 1, 64, 16, 64, True, False, 0),
    ([33, 2], [100, 2], 4, 4, 128, 8, 64, True, True, 0),
    ([33, 2], [100, 2], 4, 4, 128, 1, 24, False, True, 0),
    ([9], [1000000], 2, 2, 256, 1024, 256, False, True, 990000),
    ([3, 4], [40, 2], 16, 1, 64, 16, 8, True, False, 38),       # tokens in the prefix and before position 0
    ([6], [30], 3, 3, 256, 4, 0, False, True, 0),               # no rotation
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append_against_oracle(i, dtype):
    """Off by the output's rounding; the angle is exact to fp32 sine and cosine (2^-22 of the pair's
    length with magnitude 1, 2^-21 with the norm's factor)."""
    q_lens, kv_lens, Hq, Hkv, D, page, rot, inter, norm, prefix = APPENDS[i]
    cache, batch, table, kv0, q, k, v = _append_case(q_lens, kv_lens, Hq, Hkv, D, page, dtype, prefix, seed=i)
    g = np.random.default_rng(100 + i)
    freq, _ = cl.rope_frequencies(rot, 500000.0) if rot else (None, 1.0)
    mag = 1.25 if i % 2 else 1.0
    rope = cl.Rope(freq.cuda(), inter, mag) if rot else None
    qw, kw = (rnd(g, (D,), dtype), rnd(g, (D,), dtype)) if norm else (None, None)
    q_out = cl.kv_append(cache, batch, k.cuda(), v.cuda(), q=q.cuda(), rope=rope, eps=1e-5,
                         q_norm=None if qw is None else qw.cuda(), k_norm=None if kw is None else kw.cuda())
    torch.cuda.synchronize()
    want_k, want_v = kv0[0].double().numpy(), kv0[1].double().numpy()
    want_q, t = np.zeros((sum(q_lens), Hq, D)), 0
    fr = [] if freq is None else freq.double().numpy()
    for b, (a, n) in enumerate(zip(q_lens, kv_lens)):
        for j in range(a):
            p = n - a + j
            x, y = q[t].double().numpy(), k[t].double().numpy()
            if norm:
                x, y = layer.head_norm(x, qw.double().numpy(), 1e-5), layer.head_norm(y, kw.double().numpy(), 1e-5)
            want_q[t] = layer.rotate(x, p, fr, inter, mag if rot else 1.0)
            if p >= prefix:
                pg, row = table[b, (p - prefix) // page], (p - prefix) % page
                want_k[pg, :, row] = layer.rotate(y, p, fr, inter, mag if rot else 1.0)
                want_v[pg, :, row] = v[t].double().numpy()
            t += 1
    u = UNIT_ROUNDOFF[dtype]
    for got, want in ((q_out, want_q), (cache.k, want_k)):
        got = out_to_numpy(got)
        size = np.linalg.norm(want, axis=-1, keepdims=True)
        assert (np.abs(got - want) <= u * np.abs(want) * 1.001 + 2.0 ** -20 * size + 2.0 ** -25).all()
    assert torch.equal(cache.v.cpu(), torch.from_numpy(want_v).to(dtype))


def test_append_strided_views_positions_and_no_query():
    cache, batch, table, _, q, k, v = _append_case([3, 20], [50, 33], 4, 2, 128, 16, F16, seed=5)
    fused = torch.cat([x.reshape(23, -1) for x in (q, k, v)], 1).cuda()
    odd = torch.empty((23, fused.shape[1] + 1), dtype=F16, device="cuda")       # rows of an odd stride
    odd[:, 1:] = fused
    freq = cl.rope_frequencies(128)[0].cuda()
    pos = torch.arange(23, dtype=torch.int32, device="cuda") * 7
    results = []
    for src in (fused, odd[:, 1:]):
        for c in (cache.k, cache.v):
            c.zero_()
        qv, kv, vv = (src[:, a:b].unflatten(1, (-1, 128)) for a, b in ((0, 512), (512, 768), (768, 1024)))
        qo = cl.kv_append(cache, batch, kv, vv, q=qv, rope=cl.Rope(freq), positions=pos)
        results.append([qo, cache.k.clone(), cache.v.clone()])
    assert cl.kv_append(cache, batch, kv, vv, rope=cl.Rope(freq), positions=pos) is None
    results.append([results[0][0], cache.k.clone(), cache.v.clone()])
    inplace = q.cuda()
    assert cl.kv_append(cache, batch, k.cuda(), v.cuda(), q=inplace, rope=cl.Rope(freq), positions=pos, q_out=inplace) is inplace
    results.append([inplace, cache.k, cache.v])
    torch.cuda.synchronize()
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))
    want = layer.rotate(q[11].double().numpy(), 77, freq.double().cpu().numpy())
    assert np.abs(out_to_numpy(results[0][0][11]) - want).max() <= 2.0 ** -11 * np.abs(want).max() + 1e-5


def test_append_skips_pages_outside_the_pool():
    cache, batch, table, kv0, q, k, v = _append_case([1, 1], [20, 20], 2, 2, 64, 16, F16)
    batch.page_table[0, 1] = cache.num_pages
    batch.page_table[1, 1] = -1
    cl.kv_append(cache, batch, k.cuda(), v.cuda())
    torch.cuda.synchronize()
    assert torch.equal(cache.k.cpu(), kv0[0]) and torch.equal(cache.v.cpu(), kv0[1])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_append_leaves_rows_of_no_sequence_alone(norm, in_place):
    """Tokens ahead of the first sequence, between q_start's last entry and the end, and past a start that was
    cut: their queries are not written, and the caches hold nothing of them."""
    cache, batch, _, kv0, q, k, v = _append_case([2, 3], [40, 50], 4, 2, 64, 16, F16)
    g = np.random.default_rng(8)
    pad = lambda t: torch.cat([rnd(g, (1, *t.shape[1:]), F16), t, rnd(g, (2, *t.shape[1:]), F16)]).cuda()  # noqa: E731
    qd, kd, vd = pad(q), pad(k), pad(v)
    wide = cl.KvBatch(batch.kv_len, batch.page_table, 8, q_len=3, q_start=i32([1, 3, 6]), max_kv_len=50)
    args = dict(rope=cl.Rope(cl.rope_frequencies(64)[0].cuda()))
    if norm:
        args.update(q_norm=rnd(g, (64,), F16).cuda(), k_norm=rnd(g, (64,), F16).cuda())
    want = cl.kv_append(cache, batch, k.cuda(), v.cuda(), q=q.cuda(), **args)
    pools = cache.k.clone(), cache.v.clone()
    cache.k.copy_(kv0[0]), cache.v.copy_(kv0[1])
    for positions in (None, torch.full((8,), 5, dtype=torch.int32, device="cuda")):
        out = qd.clone() if in_place else torch.full_like(qd, 7.0)
        before = out.clone()
        cl.kv_append(cache, wide, kd, vd, q=out if in_place else qd, q_out=out, positions=positions, **args)
        torch.cuda.synchronize()
        assert torch.equal(out[0], before[0]) and torch.equal(out[6:], before[6:])
        if positions is None:
            assert torch.equal(out[1:6], want) and torch.equal(cache.k, pools[0]) and torch.equal(cache.v, pools[1])


# ---------------------------------------------------------------------- route

ROUTES = [
    # T, E, k, score, groups, top, group_best, bias, renormalize, dtype
    (1, 128, 8, "softmax", 1, 1, 1, False, True, F32),
    (64, 128, 8, "softmax", 1, 1, 1, False, True, F16),
    (7, 1, 1, "softmax", 1, 1, 1, False, False, F32),
    (33, 60, 4, "sigmoid", 1, 1, 1, False, True, BF16),
    (301, 256, 8, "sigmoid", 8, 4, 2, True, True, F32),
    (20, 256, 6, "sigmoid", 8, 3, 2, False, False, F32),
    (20, 1024, 64, "softmax", 64, 9, 1, False, True, F32),
    (5, 77, 77 // 2, "softmax", 7, 5, 1, True, True, F32),
    (50, 320, 10, "softmax", 4, 2, 2, False, True, BF16),
    (2, 1000, 3, "sigmoid", 1, 1, 1, True, True, F16),
]


@pytest.mark.parametrize("i", range(len(ROUTES)))
def test_route_against_oracle(i):
    T, E, k, score, groups, top, best, bias, renorm, dtype = ROUTES[i]
    g = np.random.default_rng(i)
    logits = rnd(g, (T, E), dtype, 2.0)
    b = rnd(g, (E,), F32, 0.1) if bias else None
    ranks = [g.integers(0, 33, E) for _ in range(i % 4)]
    levels = (0, 8, 16, 32)
    r = cl.Router(E, k, score, None if b is None else b.cuda(), groups, top, best, renorm, 1.5)
    got = cl.moe_route(r, logits.cuda(), [i32(x) for x in ranks], levels if ranks else ())
    torch.cuda.synchronize()
    ids, w = got[0].cpu().numpy(), got[1].double().cpu().numpy()
    rid, rw, gap = layer.route(logits.double().numpy(), k, score, None if b is None else b.double().numpy(), groups, top,
                               best, renorm, 1.5)
    # equal logits tie exactly (gap 0) and must go to the lower id; gaps below fp32's reach may go either way
    sure = (gap > 1e-5) | ((gap == 0) & (b is None) & (best == 1))
    assert sure.mean() > 0.5 and np.array_equal(ids[sure], rid[sure])
    assert all(len(set(row)) == k and 0 <= min(row) and max(row) < E for row in ids.tolist())
    assert (np.abs(w - rw)[sure] <= 4e-6 * np.abs(rw[sure]) + 1e-9).all()
    if ranks:
        for table, x in zip(got[2], ranks):
            assert np.array_equal(table.cpu().numpy(), wl.dynamic_slot_ranks(ids, got[1].cpu().numpy(), x, levels, 32))


@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,top,k", [(64, 64, 8, 8), (64, 64, 9, 4), (7, 7, 3, 3), (48, 24, 5, 6)])
def test_route_by_two_best_of_groups_of_one_and_two_experts(E, groups, top, k, score, bias):
    """A group of one has one best score, which then is its sum."""
    g = np.random.default_rng(E + top)
    logits = rnd(g, (40, E), F32, 2.0)
    b = rnd(g, (E,), F32, 0.1) if bias else None
    ids, w = cl.moe_route(cl.Router(E, k, score, None if b is None else b.cuda(), groups, top, 2), logits.cuda())
    torch.cuda.synchronize()
    rid, rw, gap = layer.route(logits.double().numpy(), k, score, None if b is None else b.double().numpy(), groups, top, 2)
    sure = gap > 1e-5
    assert sure.mean() > 0.5 and np.array_equal(ids.cpu().numpy()[sure], rid[sure])
    assert (np.abs(w.double().cpu().numpy() - rw)[sure] <= 4e-6 * np.abs(rw[sure]) + 1e-9).all()


def test_route_ties_infinities_and_nan():
    E = 130
    x = torch.zeros((6, E))
    x[1, 100:] = 1.0
    x[2] = -math.inf
    x[3, :120] = -math.inf
    x[4, 3] = math.nan
    x[5, 128:] = math.inf
    ids, w = cl.moe_route(cl.Router(E, 5), x.cuda())
    torch.cuda.synchronize()
    ids, w = ids.cpu(), w.cpu()
    assert ids[0].tolist() == [0, 1, 2, 3, 4] and torch.allclose(w[0], torch.full((5,), 0.2))
    assert ids[1].tolist() == [100, 101, 102, 103, 104]
    assert ids[2].tolist() == [0, 1, 2, 3, 4] and (w[2] == 0).all()
    assert ids[3].tolist() == [120, 121, 122, 123, 124] and torch.allclose(w[3], torch.full((5,), 0.2))
    assert 3 not in ids[4].tolist() and w[4].isnan().all()
    assert ids[5].tolist() == [128, 129, 0, 1, 2] and w[5].isnan().any()
    ids, w = cl.moe_route(cl.Router(E, 64, groups=2, top_groups=1), x[4:5].cuda())
    torch.cuda.synchronize()
    assert ids[0].tolist() == [e for e in range(65) if e != 3]         # equal groups: the lower one
    ids, _ = cl.moe_route(cl.Router(4, 4), torch.tensor([[math.nan, 1.0, -math.inf, 2.0]]).cuda())
    assert ids[0].tolist() == [3, 1, 2, 0]                     # NaN last, -inf before it


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("at", [0, 3, 129])
def test_route_with_a_bias_takes_a_nan_logit_last(at, score):
    """By softmax every score is NaN then, and equal in that: the lower ids, and the NaN logit behind them all."""
    x = torch.linspace(2.0, -2.0, 130).repeat(2, 1)
    x[0, at] = math.nan
    bias = torch.zeros(130)
    want = [e for e in range(130) if e != at]
    ids, w = cl.moe_route(cl.Router(130, 6, score, bias.cuda()), x.cuda())
    some, _ = cl.moe_route(cl.Router(5, 5, score, bias[:5].cuda()), x[:1, [at, 7, 8, 9, 10]].cuda())
    torch.cuda.synchronize()
    assert ids[0].tolist() == want[:6] and ids[1].tolist() == [0, 1, 2, 3, 4, 5] and some[0].tolist() == [1, 2, 3, 4, 0]
    assert w[0].isnan().all() if score == "softmax" else w[0].isfinite().all()


def test_route_scores_are_the_plain_ones_bit_for_bit():
    """The biased choice compares fp32 sums, so ids agree with torch's where its operations round alike."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((4096, 256), device="cuda", generator=g)
    bias = torch.randint(-60, 61, (256,), device="cuda", generator=g).float() * 0.001
    ids, _ = cl.moe_route(cl.Router(256, 8, "sigmoid", bias), x)
    want = (1 / (1 + torch.exp(-x)) + bias).sort(dim=1, descending=True, stable=True).indices[:, :8]
    assert torch.equal(ids.long(), want)


# ----------------------------------------------------------------------- norm

NORMS = [
    # T, d, slots, y, res, w, out, kind, post, gate, bias, alpha, beta
    (1, 4096, 0, F16, F16, F16, F16, "rms", False, None, False, 1.0, 1.0),
    (3, 2048, 8, F16, BF16, F32, F16, "rms", False, None, False, 1.0, 1.0),
    (5, 1000, 0, BF16, F32, BF16, BF16, "layer", True, "token", True, 0.5, 2.0),
    (2, 1001, 3, F32, F16, F16, F32, "layer", True, "channel", True, 1.0, 0.1),
    (300, 1, 0, F16, F16, F16, F16, "rms", True, None, False, 1.0, 1.0),
    (4, 8192, 2, BF16, BF16, BF16, BF16, "rms", True, "token", False, 1.0, -1.0),
    (2, 16384, 0, F16, None, F16, BF16, "layer", False, "channel", False, 1.0, 1.0),
    (2, 32768, 1, F16, F32, F32, F32, "rms", True, None, True, 1.0, 1.0),
    (1, 32767, 0, BF16, BF16, F32, BF16, "layer", True, None, False, 2.0, 1.0),
    (3, 4097, 64, F16, F16, F16, F16, "rms", False, None, False, 1.0, 1.0),
    (2, 520, 0, F32, F32, F32, F32, "layer", False, None, True, 0.0, 1.0),
]


@pytest.mark.parametrize("i", range(len(NORMS)))
def test_residual_norm_against_oracle(i):
    """fp32 sums of d (and slots) terms: at most (d / threads + 16) roundings of 2^-24 to a statistic, taken as
    2^-17 of the row's scale; then the output's rounding."""
    T, d, slots, yt, rt, wt, ot, kind, post, gate, bias, alpha, beta = NORMS[i]
    g = np.random.default_rng(i)
    y = rnd(g, (T, slots, d) if slots else (T, d), yt)
    sw = rnd(g, (T, slots), F32).abs() if slots else None
    res = None if rt is None else rnd(g, (T, d), rt, 3.0)
    w, pw, bs = rnd(g, (d,), wt), rnd(g, (d,), wt) if post else None, rnd(g, (d,), wt) if bias else None
    gt = None if gate is None else rnd(g, (T, d) if gate == "token" else (d,), wt)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    dbl = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    h, out = cl.residual_norm(dev(y), dev(w), dev(res), dev(sw), dev(pw), dev(gt), dev(bs), kind, 1e-5, alpha, beta,
                              out_dtype=ot)
    torch.cuda.synchronize()
    rh, ro = layer.residual_norm(dbl(y), dbl(w), dbl(res), dbl(sw), dbl(pw), dbl(gt), dbl(bs), kind, 1e-5, alpha, beta)
    for got, want in ((h, rh), (out, ro)):
        rms = np.sqrt(np.mean(want * want, axis=1, keepdims=True)) + np.abs(want).max(axis=1, keepdims=True)
        assert (np.abs(out_to_numpy(got) - want) <= UNIT_ROUNDOFF[got.dtype] * np.abs(want) * 1.001 + 2.0 ** -17 * rms
                + 2.0 ** -25).all()


def test_residual_norm_unaligned_rows_in_place_and_alone():
    g = np.random.default_rng(1)
    y, res, w = rnd(g, (4, 512), F16).cuda(), rnd(g, (4, 512), F16).cuda(), rnd(g, (512,), F16).cuda()
    h, out = cl.residual_norm(y, w, res)
    odd = torch.empty(4 * 512 + 1, dtype=F16, device="cuda")[1:].view(4, 512)       # 2-byte aligned
    odd.copy_(y)
    h2, out2 = cl.residual_norm(odd, w, res)
    alone = cl.residual_norm(y, w, res, h=False)
    stream = res.clone()
    h3, out3 = cl.residual_norm(y, w, stream, h=stream)
    torch.cuda.synchronize()
    assert torch.equal(h, h2) and (out.float() - out2.float()).abs().max() <= 2.0 ** -10 * out.float().abs().max()
    assert torch.equal(alone, out) and h3 is stream and torch.equal(h3, h) and torch.equal(out3, out)


def test_residual_norm_of_zeros_and_infinities():
    z = torch.zeros((2, 256), dtype=F16, device="cuda")
    w = torch.ones(256, dtype=F16, device="cuda")
    h, out = cl.residual_norm(z, w, z, kind="layer", eps=1e-6)
    y = z.clone()
    y[1, 7] = math.inf
    h2, out2 = cl.residual_norm(y, w, z)
    torch.cuda.synchronize()
    assert (h == 0).all() and (out == 0).all()
    assert (out2[0] == 0).all() and h2[1, 7] == math.inf and out2[1].isnan().any()


# ------------------------------------------- more than 2^32 work items a launch

def test_append_of_more_than_2_24_tokens():
    n = (1 << 24) + 1
    pages = n // 1024 + 1
    cache = cl.KvCache.empty(pages, 1024, 1, 64)
    k = torch.randint(-100, 100, (n, 1, 64), dtype=torch.int8, device="cuda").half()
    v = -k
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    cl.kv_append(cache, cl.KvBatch(i32([n]), table, n, q_len=n, max_kv_len=n), k, v)
    torch.cuda.synchronize()
    for got, want in ((cache.k, k), (cache.v, v)):
        assert torch.equal(got.view(-1, 64)[:n], want[:, 0])


def test_norm_and_route_of_more_than_2_26_tokens():
    n = (1 << 26) + 5
    y = torch.randint(0, 2, (n, 1), dtype=torch.int8, device="cuda").half() * 2 - 1
    out = cl.residual_norm(y, torch.ones(1, dtype=F16, device="cuda"), h=False, eps=0.0)
    ids, w = cl.moe_route(cl.Router(2, 1), torch.cat([torch.zeros_like(y), y], 1))
    torch.cuda.synchronize()
    assert torch.equal(out, y) and torch.equal(ids, (y > 0).int()) and (w == 1).all()
