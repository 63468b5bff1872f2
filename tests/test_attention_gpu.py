"""cl_attention against the fp64 oracle, through the paged cache.

Every cache row that belongs to no key of the batch holds NaN in k and v, so a
kernel that reads past a length, into another page or past a table shows it.

Tolerances, from the arithmetic: products of 16-bit values are exact in fp32 and
summed there, so a score is off by at most D 2^-24 scale sum|q k|, which moves a
probability by that much relative to itself; probabilities are rounded once to
the cache's type (u_p; fp16 ones below 2^-14 to multiples of 2^-24 instead), and
sums of n terms in fp32 lose at most n 2^-24.  With A = sum p |v| / sum p an
element is off by at most A times these, plus the output's own rounding."""

import numpy as np
import pytest
import torch

from oracle import layer
from paper_2605_05819_amd import cl
from tests.helpers import UNIT_ROUNDOFF, out_to_numpy

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


class Case:
    """A batch with its own pages in a pool of NaN, and the oracle's view of it."""

    def __init__(self, q_lens, kv_lens, Hq, Hkv, D, page, dtype, prefix=0, seed=0, uniform=False, spare=3, kstd=1.0):
        g = np.random.default_rng(seed)
        rnd = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).to(dtype)  # noqa: E731
        self.q_lens, self.kv_lens, self.Hq, self.Hkv, self.D, self.dtype = q_lens, kv_lens, Hq, Hkv, D, dtype
        B, self.prefix = len(q_lens), prefix
        self.N = sum(q_lens)
        own = [max(0, n - prefix) for n in kv_lens]
        need = [-(-n // page) for n in own]
        shared = -(-prefix // page)
        total = sum(need) + shared + spare
        pool = g.permutation(total).astype(np.int32)
        width = max(need + [1]) + 1
        table = np.full((B, width), -1, np.int32)        # entries past the keys are not read
        k = torch.full((total, Hkv, page, D), float("nan"), dtype=dtype)
        v = torch.full((total, Hkv, page, D), float("nan"), dtype=dtype)
        kp, vp = rnd(Hkv, prefix, D) * kstd, rnd(Hkv, prefix, D)
        for j in range(prefix):
            k[pool[j // page], :, j % page], v[pool[j // page], :, j % page] = kp[:, j], vp[:, j]
        at, self.ks, self.vs = shared, [], []
        for b in range(B):
            table[b, :need[b]] = pool[at:at + need[b]]
            kb, vb = rnd(Hkv, own[b], D) * kstd, rnd(Hkv, own[b], D)
            for j in range(own[b]):
                k[pool[at + j // page], :, j % page], v[pool[at + j // page], :, j % page] = kb[:, j], vb[:, j]
            at += need[b]
            n = min(kv_lens[b], prefix)
            self.ks.append(torch.cat([kp[:, :n], kb], 1).double().numpy())
            self.vs.append(torch.cat([vp[:, :n], vb], 1).double().numpy())
        self.q = rnd(max(self.N, 1), Hq, D)
        i32 = lambda a: torch.tensor(np.asarray(a, np.int32)).cuda()  # noqa: E731
        self.cache = cl.KvCache(k.cuda(), v.cuda())
        start = np.concatenate([[0], np.cumsum(q_lens)])
        self.table = i32(table)
        self.batch = cl.KvBatch(i32(kv_lens), self.table, max(self.N, 1), q_len=max(q_lens + [1]),
                                q_start=None if uniform else i32(start), max_kv_len=max(kv_lens + [1]),
                                prefix_table=i32(pool[:shared]) if prefix else None, prefix_len=prefix)

    def oracle(self, scale, causal, window):
        parts, at = [], 0
        for b, a in enumerate(self.q_lens):
            parts.append(layer.attend(self.q[at:at + a].double().numpy(), self.ks[b], self.vs[b], scale, causal, window))
            at += a
        return [np.concatenate([p[i] for p in parts]) for i in range(4)]


def check(c, causal=True, window=0, out_dtype=None, scale=None, q=None):
    out_dtype = out_dtype or c.dtype
    s = c.D ** -0.5 if scale is None else scale
    lse = torch.full((max(c.N, 1), c.Hq), 7.0, device="cuda")
    out = torch.full((max(c.N, 1), c.Hq, c.D), 7.0, dtype=out_dtype, device="cuda")
    r = cl.attention(c.cache, c.batch, c.q.cuda() if q is None else q, scale=scale, causal=causal, window=window,
                     out=out, lse=lse)
    torch.cuda.synchronize()
    assert r is out
    if c.N == 0:
        return
    ref, rlse, A, most = c.oracle(s, causal, window)
    n = max(c.kv_lens)
    rel = 2.0 ** -24 * (2 * c.D * most + 2 * n + 16) + 2.0 ** -21
    up = UNIT_ROUNDOFF[c.dtype]
    allow = UNIT_ROUNDOFF[out_dtype] * np.abs(ref) * 1.01 + A * (up + rel[..., None]) * 1.01
    if c.dtype == F16:
        # n probabilities off by 2^-25 at most, over a sum of at least 1
        allow = allow + 2.0 ** -25 * n * max([np.abs(v).max(initial=0) for v in c.vs])
    got = out_to_numpy(out)
    bad = np.abs(got - ref) > allow
    assert np.isfinite(got).all() and not bad.any(), (np.abs(got - ref) / np.maximum(allow, 1e-30)).max()
    gl = lse.double().cpu().numpy()
    empty = np.isneginf(rlse)
    assert np.array_equal(np.isneginf(gl), empty) and (got[empty] == 0).all()
    err = np.abs(gl[~empty] - rlse[~empty])
    assert (err <= (2 * rel + 2.0 ** -22 * np.abs(rlse))[~empty]).all(), err.max()


SHAPES = [
    # q_lens, kv_lens, Hq, Hkv, D, page, prefix
    ([1], [1], 4, 4, 64, 16, 0),
    ([1], [257], 8, 2, 128, 16, 0),
    ([1, 1, 1], [1, 33, 700], 32, 8, 128, 64, 0),
    ([1, 1], [64, 65], 7, 1, 128, 8, 0),
    ([1, 1, 1, 1], [0, 5, 31, 32], 16, 1, 64, 1, 0),          # a sequence without keys, pages of one key
    ([1] * 5, [130, 1, 90, 511, 512], 6, 2, 256, 32, 0),
    ([4, 4], [300, 77], 8, 2, 128, 16, 0),                     # drafted tokens
    ([8, 8], [1000, 9], 32, 2, 64, 64, 0),                     # 128 rows a key head
    ([5], [3], 4, 2, 128, 16, 0),                              # more new tokens than keys: the first see none
    ([65], [65], 4, 1, 128, 16, 0),                            # prompts
    ([200, 0, 17, 1], [200, 40, 100, 333], 8, 2, 128, 16, 0),
    ([129, 64], [300, 64], 3, 3, 64, 64, 0),
    ([77, 130], [80, 200], 4, 4, 256, 128, 0),
    ([0, 0], [5, 0], 4, 4, 64, 16, 0),
    ([300], [1024], 14, 2, 64, 1024, 0),
    ([1] * 6, [100, 101, 133, 300, 164, 100], 8, 2, 128, 16, 100),     # a shared prefix, odd and even pages
    ([1] * 20, [256 + 3 * i for i in range(20)], 32, 8, 128, 64, 256),
    ([3, 2, 1], [520, 515, 514], 16, 2, 64, 32, 513),
    ([40, 7], [400, 300], 4, 1, 256, 64, 290),
    ([1] * 3, [20, 700, 0], 8, 8, 128, 16, 600),               # shorter than the prefix, and empty
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_oracle(shape, dtype):
    q, kv, Hq, Hkv, D, page, prefix = SHAPES[shape]
    c = Case(q, kv, Hq, Hkv, D, page, dtype, prefix, seed=shape)
    check(c)
    check(c, causal=False, out_dtype=F32)


@pytest.mark.parametrize("window", [1, 2, 33, 100, 5000])
@pytest.mark.parametrize("shape", [2, 6, 10, 12, 17])
def test_window(shape, window):
    q, kv, Hq, Hkv, D, page, prefix = SHAPES[shape]
    c = Case(q, kv, Hq, Hkv, D, page, BF16 if shape % 2 else F16, prefix, seed=shape)
    check(c, window=window)
    check(c, window=window, causal=False)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_keys_are_split_and_joined(D):
    c = Case([1, 2], [9001, 4097], 8, 2, D, 64, F16, seed=D)
    check(c)
    c = Case([1] * 4, [6000, 6100, 5555, 7000], 8, 2, D, 32, BF16, prefix=5555, seed=D)
    check(c, out_dtype=F32)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_lengths_around_tiles(n):
    check(Case([1], [n], 4, 2, 128, 16, F16, seed=n))
    check(Case([n], [n], 2, 1, 128, 16, BF16, seed=n))
    check(Case([n], [n + 40], 1, 1, 64, 32, F16, seed=n))


def test_uniform_batches_need_no_starts():
    check(Case([3] * 4, [10, 500, 3, 129], 8, 2, 128, 16, F16, uniform=True))
    check(Case([1] * 4, [10, 500, 3, 129], 8, 2, 128, 16, BF16, uniform=True))


def test_sharp_scores_and_other_scales():
    """Scores in the hundreds: the largest dominates and nothing overflows."""
    c = Case([1, 30], [700, 300], 8, 2, 128, 16, F16, kstd=8.0)
    check(c, scale=1.0)
    check(c, scale=-0.5)
    check(c, scale=0.0)


def test_fused_projection_views():
    """q as a view of a wider row: its tokens at a stride of their own."""
    c = Case([2, 40], [100, 60], 8, 2, 128, 16, F16)
    wide = torch.full((c.N, 8 * 128 + 2 * 2 * 128), float("nan"), dtype=F16, device="cuda")
    wide[:, :8 * 128] = c.q.cuda().reshape(c.N, -1)
    check(c, q=wide[:, :8 * 128].view(c.N, 8, 128))


def test_rows_of_no_sequence_are_left_alone():
    c = Case([2, 3], [40, 50], 4, 2, 64, 16, F16)
    start = torch.tensor([1, 3, 6], dtype=torch.int32, device="cuda")
    b = cl.KvBatch(c.batch.kv_len, c.table, 8, q_len=3, q_start=start, max_kv_len=50)
    q = torch.zeros((8, 4, 64), dtype=F16, device="cuda")
    q[1:6] = c.q.cuda()
    out = torch.full((8, 4, 64), 7.0, dtype=F32, device="cuda")
    cl.attention(c.cache, b, q, out=out)
    want = cl.attention(c.cache, c.batch, c.q.cuda(), out_dtype=F32)
    torch.cuda.synchronize()
    assert torch.equal(out[1:6], want) and (out[0] == 7).all() and (out[6:] == 7).all()


def test_pages_outside_the_pool_give_nan_and_touch_nothing_else():
    c = Case([1, 1, 20], [100, 100, 100], 4, 2, 64, 16, F16)
    good = cl.attention(c.cache, c.batch, c.q.cuda())
    for bad in (-1, c.cache.num_pages, 1 << 30):
        c.table[1, 3] = bad
        out = cl.attention(c.cache, c.batch, c.q.cuda())
        torch.cuda.synchronize()
        assert out[1].isnan().all() and torch.equal(out[0], good[0]) and torch.equal(out[2:], good[2:])


def test_lengths_beyond_the_bounds_are_cut():
    """A kv_len past max_kv_len or the table, and starts past the tokens, stay inside what the host gave."""
    c = Case([1, 1], [64, 64], 4, 2, 64, 16, F16, spare=0)
    want = cl.attention(c.cache, c.batch, c.q.cuda())
    wide = cl.KvBatch(torch.tensor([1 << 30, 64], dtype=torch.int32, device="cuda"), c.table[:, :4].contiguous(), 2,
                      q_start=torch.tensor([0, 1, 999], dtype=torch.int32, device="cuda"))
    got = cl.attention(c.cache, wide, c.q.cuda())
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_results_repeat_bit_for_bit_and_on_other_streams():
    c = Case([1, 3, 50], [5000, 3000, 400], 8, 2, 128, 16, BF16, prefix=300)
    q = c.q.cuda()
    want = cl.attention(c.cache, c.batch, q, out_dtype=F32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        assert torch.equal(cl.attention(c.cache, c.batch, q, out_dtype=F32), want)
        with torch.cuda.stream(side):
            x = q + 0
            got = cl.attention(c.cache, c.batch, x, out_dtype=F32)
        explicit = cl.attention(c.cache, c.batch, q, out_dtype=F32, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(explicit, want)


def test_a_pool_beyond_2_31_elements():
    """The last pages of a pool of 2^31 + elements: offsets pass 32 bits."""
    Hkv, page, D = 8, 64, 128
    pages = (1 << 31) // (Hkv * page * D) + 3
    k = torch.empty((pages, Hkv, page, D), dtype=F16, device="cuda")
    v = torch.empty_like(k)
    c = Case([1, 9], [150, 100], 16, Hkv, D, page, F16, spare=0)
    own = torch.arange(c.cache.num_pages, dtype=torch.int32, device="cuda")
    at = pages - c.cache.num_pages
    k[at:], v[at:] = c.cache.k[own.long()], c.cache.v[own.long()]
    table = torch.where(c.table >= 0, c.table + at, c.table)
    b = cl.KvBatch(c.batch.kv_len, table, c.N, q_len=9, q_start=c.batch.q_start, max_kv_len=150)
    got = cl.attention(cl.KvCache(k, v), b, c.q.cuda())
    want = cl.attention(c.cache, c.batch, c.q.cuda())
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_workspace_is_checked_and_sized_by_the_descriptors():
    c = Case([1], [9000], 8, 2, 128, 16, F16)
    need = cl.attention_workspace(c.cache, c.batch, 8)
    if need:
        with pytest.raises(cl.ClError) as e:
            cl.attention(c.cache, c.batch, c.q.cuda(), ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
        assert e.value.status == cl.CL_EWORKSPACE
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")     # NaN: nothing in it has to be set
    out = cl.attention(c.cache, c.batch, c.q.cuda(), ws=ws)
    torch.cuda.synchronize()
    assert out.isfinite().all() and (ws[need:] == 255).all()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("q,kv,D,window", [([4], [40], 128, 0), ([8, 3], [100, 70], 64, 20), ([130], [200], 128, 0),
                                           ([100, 40], [100, 300], 64, 33), ([90], [90], 256, 0), ([3], [600], 256, 500)])
def test_infinities_and_nan_reach_only_the_rows_that_see_them(q, kv, D, window, dtype):
    """Some keys and values of the sequences are NaN or infinite: rows that do not see them equal those of
    finite contents, rows that see a value of that kind have it in that dim, and NaN everywhere for a NaN key."""
    c = Case(q, kv, 8, 2, D, 16, dtype, seed=D + window)
    clean = cl.attention(c.cache, c.batch, c.q.cuda(), window=window, out_dtype=F32)
    bad = [(0, kv[0] - 2, "v", float("inf"), 5), (0, kv[0] - q[0] // 2 - 1, "v", float("nan"), D - 1)]
    bad += [(len(q) - 1, kv[-1] - 1, "k", float("nan"), 3), (0, max(0, kv[0] - q[0] - 10), "v", float("-inf"), 0)]
    for b, j, what, x, dim in bad:
        page = c.table[b, j // 16].long()
        getattr(c.cache, what)[page, 1, j % 16, dim] = x                          # the second key head's
    out = cl.attention(c.cache, c.batch, c.q.cuda(), window=window, out_dtype=F32)
    torch.cuda.synchronize()
    at = 0
    for b, (a, n) in enumerate(zip(q, kv)):
        for i in range(a):
            p, row, ref = n - a + i, out[at + i].cpu(), clean[at + i].cpu()
            touched = torch.zeros(8, D, dtype=torch.bool)
            for bb, j, what, x, dim in bad:
                if bb == b and j <= p and (not window or j > p - window):
                    if what == "k":
                        touched[4:] = True
                        assert row[4:].isnan().all()
                    else:
                        touched[4:, dim] = True
                        assert not row[4:, dim].isfinite().any()
            assert torch.allclose(row[~touched], ref[~touched], rtol=2.0 ** -20, atol=2.0 ** -20), (b, i)
        at += a


def test_a_stream_of_its_own_beside_a_busy_one():
    """Calls on another stream allocate for that stream: memory freed on the current one, where long work is
    still queued that reads it, is not taken for their workspace or results."""
    c = Case([1, 2, 1], [5000, 3000, 4000], 8, 2, 128, 16, F16)
    q = c.q.cuda()
    want = cl.attention(c.cache, c.batch, q, out_dtype=F32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.ones((4096, 4096), device="cuda")
    for _ in range(5):
        x = torch.full((cl.attention_workspace(c.cache, c.batch, 8) // 4,), 3.0, device="cuda")
        for _ in range(20):
            big = (big @ big).clamp_(max=1.0)
        keep = x * 2                                   # queued behind the products
        del x                                          # its memory is free for the current stream
        got = cl.attention(c.cache, c.batch, q, out_dtype=F32, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool((keep == 6.0).all())


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("n", [2, 31, 32, 33, 64, 200, 3000])
def test_tokens_past_q_len_hide_their_keys_from_the_one_attended(n, dtype):
    """q_len 1 and a range of three tokens: the first alone is attended for, and it does not see the last two
    keys, whose values (and one key) are infinite and NaN."""
    c = Case([1], [n], 8, 2, 128, 16, dtype, seed=n)
    room = torch.cat([c.table, torch.full((1, 2), -1, dtype=torch.int32, device="cuda")], 1)
    used = set(room[0].tolist())
    spare = [p for p in range(c.cache.num_pages) if p not in used]
    for j, bad in ((n, float("nan")), (n + 1, float("inf"))):
        if room[0, j // 16] < 0:
            room[0, j // 16] = spare.pop()
        page = room[0, j // 16].long()
        c.cache.k[page, :, j % 16], c.cache.v[page, :, j % 16] = 1.0, bad
    c.cache.k[page, 1, j % 16, 0] = float("nan")
    b = cl.KvBatch(torch.tensor([n + 2], dtype=torch.int32, device="cuda"), room, 3, q_len=1,
                   q_start=torch.tensor([0, 3], dtype=torch.int32, device="cuda"), max_kv_len=n + 2)
    out = torch.full((3, 8, 128), 7.0, device="cuda")
    cl.attention(c.cache, b, torch.cat([c.q, c.q * 2, c.q * 3]).cuda(), out=out)
    torch.cuda.synchronize()
    ref, _, A, most = c.oracle(128 ** -0.5, True, 0)
    allow = A * (UNIT_ROUNDOFF[dtype] + 2.0 ** -24 * (2 * 128 * most + 2 * n + 16)[..., None] + 2.0 ** -21) * 1.01
    allow = allow + (2.0 ** -25 * n * np.abs(c.vs[0]).max() if dtype == F16 else 0)
    assert (np.abs(out_to_numpy(out[:1]) - ref) <= allow).all() and (out[1:] == 7).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("q_len,kv", [(1, 9000), (3, 9000), (40, 9000), (1100, 3000)])
def test_seen_infinities_stay_in_results_of_split_keys(q_len, kv, bad):
    """A value that is not finite among keys whose whole split is e^-1024 of another: its dim is not finite,
    whichever kernel joins the splits."""
    c = Case([q_len], [kv], 4, 1, 64, 16, BF16, seed=q_len, kstd=0.0)
    j = torch.arange(kv - q_len, device="cuda")             # seen by every row
    c.cache.k[c.table[0, j // 16].long(), 0, j % 16] = -16.0
    c.cache.v[c.table[0, 0].long(), 0, 3, 11] = bad
    out = cl.attention(c.cache, c.batch, torch.ones_like(c.q).cuda(), scale=1.0, out_dtype=F32)
    torch.cuda.synchronize()
    assert not out[:, :, 11].isfinite().any() and out[:, :, :11].isfinite().all() and out[:, :, 12:].isfinite().all()


class Tail:
    """One sequence of n keys of one head, of which every `every`-th from the first is a sink that all queries
    score 0, and the others -low to -high; values of one sign, 0 at the sinks."""

    def __init__(self, a, n, every, low, high, D, dtype, prefix=0):
        g = np.random.default_rng(n + a + D)
        sink = np.arange(n) % every == 0
        k = np.zeros((n, D))
        k[:, 0] = np.where(sink, 0.0, -g.uniform(low, high, n))
        v = np.where(sink[:, None], 0.0, g.uniform(0.5, 1.0, (n, D)))
        k, v = (torch.from_numpy(x).to(dtype) for x in (k, v))
        self.a, self.n, self.sinks = a, n, sink
        q = torch.zeros((a, 1, D), dtype=dtype)
        q[:, :, 0] = 1.0
        page, pages = 64, -(-n // 64)
        pool = torch.zeros((2, pages * page, D), dtype=dtype)
        pool[0, :n], pool[1, :n] = k, v
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.cache = cl.KvCache(*(x.view(pages, 1, page, D).cuda() for x in pool))
        table = torch.arange(pages, dtype=torch.int32, device="cuda")
        shared = prefix // page
        self.batch = cl.KvBatch(i32([n]), table[None, shared:].contiguous(), a, q_len=a, max_kv_len=n,
                                prefix_table=table[:shared].contiguous() if shared else None, prefix_len=shared * page)
        self.q, self.k, self.v = q, k.double().numpy(), v.double().numpy()

    def check(self, dtype):
        lse = torch.empty((self.a, 1), device="cuda")
        out = cl.attention(self.cache, self.batch, self.q.cuda(), scale=1.0, out_dtype=F32, lse=lse)
        torch.cuda.synchronize()
        for i in sorted({0, self.a // 2, self.a - 1}):
            see = self.n - self.a + i + 1
            p = np.exp(self.k[:see, 0])
            want = p @ self.v[:see] / p.sum()
            # every p once by the type's unit, or in fp16 by 2^-25 of 2^-12 of the maximum (1, and one sink at least
            # is in the sum); scores of one exact product; a lane sums see / 4 terms at most
            allow = want * (UNIT_ROUNDOFF[dtype] + 2.0 ** -24 * (see / 4 + 64)) * 1.01
            if dtype == F16:
                allow = allow + 2.0 ** -37 * see / self.sinks[:see].sum()
            err = np.abs(out[i, 0].double().cpu().numpy() - want)
            assert (err <= allow).all(), (i, (err / allow).max(), (err / want).max())
            assert abs(lse[i, 0].item() - np.log(p.sum())) <= 2.0 ** -24 * (see / 4 + 64)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("a,n", [(1, 1000), (2, 1000), (20, 1000), (40, 1500), (300, 700), (700, 2100)])
def test_small_probabilities_beside_sinks_keep_their_mass(a, n, D, dtype):
    """Keys at e^-17 to e^-20 of the largest, in every wave's share a sink: single tokens, a few, tiles of 64 and
    128 rows, in one split and in several."""
    Tail(a, n, 32, 17.0, 20.0, D, dtype).check(dtype)


@pytest.mark.parametrize("a,prefix", [(1, 0), (24, 0), (40, 0), (1, 1024), (40, 1024)])
def test_one_sink_over_a_long_diffuse_tail(a, prefix):
    Tail(a, 100001, 100001, 17.0, 19.0, 64, F16, prefix).check(F16)


def test_launches_of_more_than_2_24_workgroups():
    """A prompt beside 2048 sequences of one token: each sequence has the longest one's workgroups."""
    seqs, n, heads, D = 2049, 16384, 64, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = n // 64 + seqs - 1
    k, v = (torch.randn((pages, heads, 64, D), device="cuda", generator=g, dtype=F32).half() for _ in range(2))
    table = torch.full((seqs, n // 64), -1, dtype=torch.int32, device="cuda")
    table[0] = torch.arange(n // 64)
    table[1:, 0] = torch.arange(n // 64, pages)
    kv_len = torch.ones(seqs, dtype=torch.int32, device="cuda")
    kv_len[0] = n
    start = torch.cat([torch.zeros(1, dtype=torch.int32), torch.arange(n, n + seqs, dtype=torch.int32)]).cuda()
    q = torch.randn((n + seqs - 1, heads, D), device="cuda", generator=g).half()
    cache = cl.KvCache(k, v)
    out = cl.attention(cache, cl.KvBatch(kv_len, table, n + seqs - 1, q_len=n, q_start=start, max_kv_len=n), q)
    alone = cl.attention(cache, cl.KvBatch(kv_len[:1].contiguous(), table[:1].contiguous(), n, q_len=n, max_kv_len=n), q[:n])
    torch.cuda.synchronize()
    assert torch.equal(out[:n], alone) and torch.equal(out[n:], v[n // 64:, :, 0])      # one key: its value


def test_joins_of_more_than_2_24_rows():
    """2^25 + 2^18 rows of two splits, every sequence the same."""
    seqs, q_len, heads, D = 129, 4096, 64, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = cl.KvCache(*(torch.randn((3, 1, 64, D), device="cuda", generator=g).half() for _ in range(2)))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    one = torch.randn((q_len, heads, D), device="cuda", generator=g).half()
    batch = lambda n: cl.KvBatch(i32(*[80] * n), i32(*[[1]] * n), n * q_len, q_len=q_len, max_kv_len=80,  # noqa: E731
                                 prefix_table=i32(2), prefix_len=64)
    out = cl.attention(cache, batch(seqs), one.repeat(seqs, 1, 1), causal=False).view(seqs, q_len, heads, D)
    alone = cl.attention(cache, batch(1), one, causal=False)
    torch.cuda.synchronize()
    assert all(torch.equal(out[i], out[0]) for i in range(seqs))
    assert (out[0].float() - alone.float()).abs().max() <= 2.0 ** -9 * cache.v.float().abs().max()
