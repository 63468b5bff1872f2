"""The cache of 8 bits: attention over it, appends to it and reads of it, against fp64.

Attention's tolerances are those of the 16-bit cache (tests/test_attention_gpu.py): the codes' values are values of
the 16-bit type exactly.  Appends: v is rounded from its own 16 bits, so its codes are the oracle's; k is rotated in
fp32 first, off by at most 2^-20 of the head's pair (an angle within 2^-23 of a turn times 2 pi, two products and a
sum; 2^-21 more of a norm), so a code stands within half a step (2^-4 of the value, 2^-10 of 2^e near zero) and that."""

import numpy as np
import pytest
import torch

from oracle import cache8, layer
from paper_2605_05819_amd import cl
from tests.test_attention_gpu import SHAPES, Case, check

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
NAME = {F16: "fp16", BF16: "bf16"}


def decoded(codes, scales, block, dtype):
    """uint8 [pages][heads][rows][dim] and scales -> values of dtype (exact)."""
    e = scales.double().repeat_interleave(block, 2)[..., None] - 127
    return (codes.view(torch.float8_e4m3fn).double() * 2.0 ** e).to(dtype)


class Case8(Case):
    """A Case whose pool holds codes; its keys and values are what they stand for."""

    def __init__(self, q_lens, kv_lens, Hq, Hkv, D, page, dtype, block=None, seed=0, **kw):
        super().__init__(q_lens, kv_lens, Hq, Hkv, D, page, dtype, seed=seed, **kw)
        block = min(page, block or (1, 4, 16, 32)[seed % 4])
        g = torch.Generator().manual_seed(seed + 1)
        parts = []
        for pool in (self.cache.k, self.cache.v):
            pool = pool.cpu().float()
            e = torch.randint(-7, -4, pool.shape[:2] + (page // block,), generator=g)
            x = pool * (2.0 ** -e.float()).repeat_interleave(block, 2)[..., None]
            parts += [x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)]
        k, ks, v, vs = parts
        self.block = block
        self.cache = cl.KvCache8(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), dtype)
        dk, dv = decoded(k, ks, block, dtype), decoded(v, vs, block, dtype)
        assert torch.equal(dk.double().nan_to_num(7.0), (k.view(torch.float8_e4m3fn).double() * 2.0 ** (ks.double().repeat_interleave(block, 2)[..., None] - 127)).nan_to_num(7.0))
        self.twin = cl.KvCache(dk.cuda(), dv.cuda())
        table = self.table.cpu()
        pre = self.batch.prefix_table.cpu() if self.prefix else None
        for b, n in enumerate(kv_lens):
            at = [(pre[j // page], j % page) if j < self.prefix else (table[b, (j - self.prefix) // page], (j - self.prefix) % page)
                  for j in range(n)]
            if n:
                p, r = torch.tensor([int(x) for x, _ in at]), torch.tensor([y for _, y in at])
                self.ks[b], self.vs[b] = (t[p, :, r].permute(1, 0, 2).double().numpy() for t in (dk, dv))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_against_oracle(shape, dtype):
    q, kv, Hq, Hkv, D, page, prefix = SHAPES[shape]
    c = Case8(q, kv, Hq, Hkv, D, page, dtype, prefix=prefix, seed=shape)
    check(c)
    check(c, causal=False, out_dtype=F32)


@pytest.mark.parametrize("window", [1, 33, 100])
@pytest.mark.parametrize("shape", [2, 6, 10, 12, 17])
def test_attention_window(shape, window):
    q, kv, Hq, Hkv, D, page, prefix = SHAPES[shape]
    c = Case8(q, kv, Hq, Hkv, D, page, BF16 if shape % 2 else F16, prefix=prefix, seed=shape)
    check(c, window=window)
    check(c, window=window, causal=False)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_long_keys_are_split_and_joined(D):
    check(Case8([1, 2], [9001, 4097], 8, 2, D, 64, F16, seed=D))
    check(Case8([1] * 4, [6000, 6100, 5555, 7000], 8, 2, D, 32, BF16, prefix=5555, seed=D), out_dtype=F32)


@pytest.mark.parametrize("n", [1, 15, 17, 31, 33, 63, 64, 65, 127, 129, 255, 257])
def test_attention_lengths_around_tiles(n):
    check(Case8([1], [n], 4, 2, 128, 16, F16, seed=n))
    check(Case8([n], [n], 2, 1, 128, 16, BF16, seed=n))
    check(Case8([n], [n + 40], 1, 1, 64, 32, F16, seed=n))


@pytest.mark.parametrize("block", [1, 2, 8, 64])
def test_attention_blocks_and_scales(block):
    check(Case8([1, 3, 70], [300, 90, 200], 8, 2, 128, 64, BF16, block=block, seed=block))
    c = Case8([1, 30], [700, 300], 8, 2, 128, 64, F16, block=block, kstd=8.0)
    check(c, scale=1.0)
    check(c, scale=-0.5)
    check(c, scale=0.0)


LONG = [                                          # prompts whose keys are converted ahead: 16 row blocks and more, 256 in all
    ([600, 17, 300, 1], [600, 400, 333, 9], 16, 4, 128, 16, 8),
    ([530, 3, 0, 520], [900, 3, 20, 520], 16, 4, 64, 64, 64),
    ([300, 290, 1, 40], [300, 512, 70, 41], 16, 4, 256, 32, 1),
    ([700, 650], [1300, 650], 24, 8, 128, 256, 32),
    ([129, 128, 1, 1], [129, 200, 1, 0], 64, 4, 64, 1, 1),
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("shape", range(len(LONG)))
def test_long_prompts(shape, dtype):
    q, kv, Hq, Hkv, D, page, block = LONG[shape]
    c = Case8(q, kv, Hq, Hkv, D, page, dtype, block=block, seed=shape)
    assert cl.attention_workspace(c.cache, c.batch, Hq) >= sum(kv) * 4 * Hkv * D
    check(c)
    check(c, causal=False, window=(0, 70, 1, 130, 33)[shape], out_dtype=F32)


@pytest.mark.parametrize("shape", [0, 2])
def test_long_prompts_with_nan_codes_and_bad_pages(shape):
    q, kv, Hq, Hkv, D, page, block = LONG[shape]
    c = Case8(q, kv, Hq, Hkv, D, page, BF16, block=block, seed=shape)
    for window in (0, 40):
        c = Case8(q, kv, Hq, Hkv, D, page, BF16, block=block, seed=shape)
        x = c.q.cuda()
        ws = torch.full((cl.attention_workspace(c.cache, c.batch, Hq),), 255, dtype=torch.uint8, device="cuda")
        clean = cl.attention(c.cache, c.batch, x, window=window, out_dtype=F32, ws=ws)
        g, j = Hq // Hkv, kv[0] - 150                  # a value of the second key head in the middle of the first prompt
        c.cache.v[c.table[0, j // page].long(), 1, j % page, 5] = 0x7f
        out = cl.attention(c.cache, c.batch, x, window=window, out_dtype=F32, ws=ws.fill_(255))
        torch.cuda.synchronize()
        pos = torch.arange(kv[0] - q[0], kv[0], device="cuda")
        sees = (pos >= j) & ((pos < j + window) if window else True)
        touched = torch.zeros_like(out, dtype=torch.bool)
        touched[:q[0], g:2 * g, 5] = sees[:, None]
        assert out[touched].isnan().all() and touched.any()
        assert torch.allclose(out[~touched], clean[~touched], rtol=2.0 ** -20, atol=2.0 ** -20)
    c = Case8(q, kv, Hq, Hkv, D, page, BF16, block=block, seed=shape)
    for bad in (-1, c.cache.num_pages, 1 << 30):
        c.table[0, 3] = bad
        out = cl.attention(c.cache, c.batch, x, out_dtype=F32, causal=False)
        torch.cuda.synchronize()
        assert out[:q[0]].isnan().all() and out[q[0]:].isfinite().all()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
def test_every_code_and_exponent_decodes_exactly(dtype):
    """One key a query sees: the output is its value, for every code and the type's exponents."""
    lo, hi = cache8.RANGE[NAME[dtype]]
    es = sorted({lo, lo + 1, lo + 5, -1, 0, 1, hi - 1, hi})
    codes = torch.arange(256, dtype=torch.uint8)[None, None, None].repeat(len(es), 1, 1, 1)
    scales = torch.tensor(es, dtype=torch.int32).add(127).to(torch.uint8)[:, None, None]
    cache = cl.KvCache8(codes.cuda(), codes.cuda(), scales.cuda(), scales.cuda(), dtype)
    n = len(es)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = cl.KvBatch(i32([1] * n), i32([[i] for i in range(n)]), n, max_kv_len=1)
    q = torch.zeros((n, 1, 256), dtype=dtype, device="cuda")
    k, v = cl.kv_read(cache, batch)
    want = cache8.decode(codes[:, 0, 0].numpy()) * 2.0 ** np.array(es)[:, None]
    big = np.abs(want) > cache8.MOST[NAME[dtype]]                 # codes that an append does not write
    for got in (k, v):
        got = got[:, 0].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want) & ~big
        assert np.array_equal(got[ok], want[ok])
    good = torch.from_numpy(~np.isnan(want[0]) & ~big[-1]).cuda()  # a NaN key gives NaN everywhere: mask it
    clean = torch.where(good, codes.cuda(), 0)
    cache = cl.KvCache8(clean, clean, scales.cuda(), scales.cuda(), dtype)
    for rows in (1, 20):                                          # a stream and a tile
        b = cl.KvBatch(batch.kv_len, batch.page_table, n * rows, q_len=rows, max_kv_len=1)
        out = cl.attention(cache, b, q.repeat_interleave(rows, 0), causal=False, out_dtype=F32).double().cpu().numpy()
        want2 = np.where(good.cpu().numpy(), np.nan_to_num(want), 0.0).repeat(rows, 0)
        assert np.array_equal(out[:, 0], want2)


@pytest.mark.parametrize("q,kv,D,window", [([4], [40], 128, 0), ([8, 3], [100, 70], 64, 20), ([130], [200], 128, 0),
                                           ([90], [90], 256, 0), ([3], [600], 256, 500)])
def test_nan_codes_reach_only_the_rows_that_see_them(q, kv, D, window):
    c = Case8(q, kv, 8, 2, D, 16, BF16, seed=D + window)
    clean = cl.attention(c.cache, c.batch, c.q.cuda(), window=window, out_dtype=F32)
    bad = [(0, kv[0] - 2, "v", 5), (0, kv[0] - q[0] // 2 - 1, "v", D - 1), (len(q) - 1, kv[-1] - 1, "k", 3)]
    for b, j, what, dim in bad:
        getattr(c.cache, what)[c.table[b, j // 16].long(), 1, j % 16, dim] = 0xff
    out = cl.attention(c.cache, c.batch, c.q.cuda(), window=window, out_dtype=F32)
    torch.cuda.synchronize()
    at = 0
    for b, (a, n) in enumerate(zip(q, kv)):
        for i in range(a):
            p, row, ref = n - a + i, out[at + i].cpu(), clean[at + i].cpu()
            touched = torch.zeros(8, D, dtype=torch.bool)
            for bb, j, what, dim in bad:
                if bb == b and j <= p and (not window or j > p - window):
                    if what == "k":
                        touched[4:] = True
                    else:
                        touched[4:, dim] = True
            assert row[touched].isnan().all()
            assert torch.allclose(row[~touched], ref[~touched], rtol=2.0 ** -20, atol=2.0 ** -20), (b, i)
        at += a


def test_pages_outside_the_pool_give_nan():
    c = Case8([1, 1, 20], [100, 100, 100], 4, 2, 64, 16, F16)
    good = cl.attention(c.cache, c.batch, c.q.cuda())
    for bad in (-1, c.cache.num_pages, 1 << 30):
        c.table[1, 3] = bad
        out = cl.attention(c.cache, c.batch, c.q.cuda())
        torch.cuda.synchronize()
        assert out[1].isnan().all() and torch.equal(out[0], good[0]) and torch.equal(out[2:], good[2:])


def test_a_pool_beyond_2_31_bytes():
    Hkv, page, D = 8, 64, 128
    pages = (1 << 31) // (Hkv * page * D) + 3
    c = Case8([1, 9], [150, 100], 16, Hkv, D, page, F16, block=16, spare=0)
    at = pages - c.cache.num_pages
    big = []
    for x in (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale):
        y = torch.empty((pages,) + x.shape[1:], dtype=torch.uint8, device="cuda")
        y[at:] = x
        big.append(y)
    table = torch.where(c.table >= 0, c.table + at, c.table)
    b = cl.KvBatch(c.batch.kv_len, table, c.N, q_len=9, q_start=c.batch.q_start, max_kv_len=150)
    got = cl.attention(cl.KvCache8(*big, F16), b, c.q.cuda())
    want = cl.attention(c.cache, c.batch, c.q.cuda())
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    new = torch.randn((c.N, Hkv, D), device="cuda").half()
    cl.kv_append(cl.KvCache8(*big, F16), b, new, new)
    cl.kv_append(c.cache, c.batch, new, new)
    torch.cuda.synchronize()
    assert all(torch.equal(y[at:], x) for x, y in zip((c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale), big))


# ------------------------------------------------------------------- appends

class Pool:
    """Sequences in a pool of random bytes, and the oracle's appends to a copy of it."""

    def __init__(self, lens, Hkv, D, page, block, dtype, prefix=0, seed=0, width=None):
        g = torch.Generator().manual_seed(seed)
        need = [-(-max(0, n - prefix) // page) for n in lens]
        self.width = width or max(need + [1])
        total = sum(need) + 4
        perm = torch.randperm(total, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        at = 1
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        rnd = lambda hi, *s: torch.randint(0, hi, s, generator=g, dtype=torch.int32).to(torch.uint8)  # noqa: E731
        self.t = [rnd(0x7f, total, Hkv, page, D), rnd(0x7f, total, Hkv, page, D), rnd(256, total, Hkv, page // block),
                  rnd(256, total, Hkv, page // block)]
        for x in self.t[2:]:
            x.copy_(x % 6 + 116)
        self.cache = cl.KvCache8(*[x.cuda() for x in self.t], dtype)
        self.lens, self.Hkv, self.D, self.page, self.block, self.dtype, self.prefix = lens, Hkv, D, page, block, dtype, prefix

    def batch(self, lens, counts, **kw):
        start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32).cuda()
        return cl.KvBatch(torch.tensor(lens, dtype=torch.int32).cuda(), self.table.cuda(), sum(counts), q_len=max(counts),
                          q_start=start, max_kv_len=max(lens), prefix_len=self.prefix,
                          prefix_table=torch.zeros(-(-self.prefix // self.page), dtype=torch.int32).cuda() if self.prefix else None, **kw)

    def check(self, lens, counts, knew, vnew, rel=2.0 ** -20):
        """self.t is the pool before the append; knew, vnew [tokens][heads][dim] fp64 values."""
        got = [x.cpu() for x in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale)]
        want = [x.clone() for x in self.t]
        at = 0
        for b, (n, a) in enumerate(zip(lens, counts)):
            i = 0
            while i < a:
                mine = n - a + i - self.prefix
                if mine < 0:
                    i += 1
                    continue
                before = mine % self.block
                run = min(self.block - before, a - i)
                page, row = int(self.table[b, mine // self.page]), mine % self.page
                if 0 <= page < len(self.t[0]):
                    for h in range(self.Hkv):
                        for w, new in ((0, knew), (1, vnew)):
                            x = new[at + i:at + i + run, h]
                            e0 = int(self.t[2 + w][page, h, row // self.block]) - 127
                            old = self.t[w][page, h, row - before:row].numpy()
                            codes, e = cache8.append(old, e0, x, NAME[self.dtype])
                            assert int(got[2 + w][page, h, row // self.block]) == e + 127
                            mine_got = got[w][page, h, row - before:row + run].numpy()
                            one = lambda x: np.where(x == 0xff, 0x7f, x)  # noqa: E731  (NaN has two codes)
                            if w == 1:
                                assert np.array_equal(one(mine_got), one(codes))
                            else:
                                assert np.array_equal(one(mine_got[:before]), one(codes[:before]))
                                v = cache8.decode(mine_got[before:]) * 2.0 ** e
                                fine = np.isfinite(x)
                                assert np.array_equal(np.isnan(v), ~fine)
                                most = cache8.MOST[NAME[self.dtype]]
                                ref = np.clip(np.where(fine, x, 0), -most, most)
                                far = np.abs(np.where(fine, x, 0)).max(axis=1, keepdims=True)
                                allow = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** (e - 10)) * (1 + 2.0 ** -10) + rel * far
                                assert (np.abs(np.where(fine, v, 0) - ref) <= allow).all()
                            want[w][page, h, row - before:row + run] = torch.from_numpy(mine_got.copy())
                            want[2 + w][page, h, row // self.block] = e + 127
                i += run
            at += a
        assert all(torch.equal(x, y) for x, y in zip(got, want))      # and nothing else changed
        self.t = got


def turned(x, lens, counts, freq, inter=False, w=None):
    out, at = np.array(x, dtype=np.float64), 0
    for n, a in zip(lens, counts):
        for i in range(a):
            h = out[at + i] if w is None else layer.head_norm(out[at + i], w, 1e-6)
            out[at + i] = h if freq is None else layer.rotate(h, n - a + i, freq, inter)
        at += a
    return out


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("D,page,block,inter,norm", [(128, 16, 16, False, False), (64, 32, 8, True, True), (256, 64, 64, False, True),
                                                     (128, 64, 1, True, False), (64, 8, 2, False, False)])
def test_append_against_oracle(D, page, block, inter, norm, dtype):
    """Prompts, then steps of a few tokens that begin in the middle of blocks, larger values among them."""
    g = np.random.default_rng(D + block)
    Hq, Hkv = 6, 2
    p = Pool([150, 60, 200], Hkv, D, page, block, dtype, seed=D)
    freq = cl.rope_frequencies(D, 10000.0)[0]
    w = torch.from_numpy(1 + 0.2 * g.standard_normal(D)).to(dtype)
    lens = np.zeros(3, np.int64)
    for step, counts in enumerate(([100, 3, 33], [1, 1, 1], [5, 1, 70], [1, 30, 2], [1, 1, 1])):
        lens += counts
        N = sum(counts)
        size = 2.0 ** g.integers(-6, 7, (N, 1, 1))
        rnd = lambda h: torch.from_numpy(g.standard_normal((N, h, D)) * size).to(dtype)  # noqa: E731
        q, k, v = rnd(Hq), rnd(Hkv), rnd(Hkv)
        rope = cl.Rope(freq.cuda(), interleaved=inter)
        out = cl.kv_append(p.cache, p.batch(list(lens), counts), k.cuda(), v.cuda(), q=q.cuda(), rope=rope,
                           q_norm=w.cuda() if norm else None, k_norm=w.cuda() if norm else None)
        torch.cuda.synchronize()
        wd = w.double().numpy() if norm else None
        p.check(lens, counts, turned(k.double().numpy(), lens, counts, freq.double().numpy(), inter, wd), v.double().numpy())
        ref = turned(q.double().numpy(), lens, counts, freq.double().numpy(), inter, wd)
        far = np.abs(ref).max(axis=-1, keepdims=True)
        u = 2.0 ** (-11 if dtype == F16 else -8)
        assert (np.abs(out.double().cpu().numpy() - ref) <= u * np.abs(ref) * 1.01 + 2.0 ** -20 * far + 2.0 ** -25).all()
        # what a read of the same batch gives is what the codes stand for
        kr, vr = cl.kv_read(p.cache, p.batch(list(lens), counts))
        val = [decoded(p.t[i], p.t[2 + i], block, dtype) for i in (0, 1)]
        at = 0
        for b, (n, a) in enumerate(zip(lens, counts)):
            for i in range(a):
                j = n - a + i
                for got, x in zip((kr, vr), val):
                    assert torch.equal(got[at + i].cpu(), x[int(p.table[b, j // page]), :, j % page])
            at += a


@pytest.mark.parametrize("D,page,block,inter,norm,prefix", [(128, 64, 16, False, True, 0), (128, 32, 32, True, False, 7), (128, 64, 64, False, False, 0),
                                                            (128, 128, 128, False, True, 100), (64, 64, 64, True, True, 0), (64, 16, 1, False, False, 0),
                                                            (256, 32, 16, False, True, 0), (256, 64, 32, True, False, 0), (64, 1024, 512, False, True, 0)])
def test_append_of_prompts(D, page, block, inter, norm, prefix):
    """Several hundred tokens at once, long and short sequences side by side, empty ones, blocks begun before and rows of no
    sequence on both sides: every block size a wave holds, and those it does not."""
    g = np.random.default_rng(D + block)
    dtype = BF16 if inter else F16
    Hkv = 3
    p = Pool([700, 40, 400, 33, 20, 1, 130], Hkv, D, page, block, dtype, prefix=prefix, seed=block)
    freq = cl.rope_frequencies(D, 10000.0)[0]
    w = torch.from_numpy(1 + 0.2 * g.standard_normal(D)).to(dtype)
    rope = cl.Rope(freq.cuda(), interleaved=inter)
    lens = np.zeros(7, np.int64)
    for counts in ([333, 0, 300, 5, 1, 0, 77], [350, 33, 1, 20, 3, 0, 40], [1, 1, 90, 0, 16, 1, 0]):
        lens += counts
        N, ahead = sum(counts), 5
        start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + ahead, dtype=torch.int32).cuda()
        pre = torch.zeros(-(-prefix // page), dtype=torch.int32).cuda() if prefix else None
        batch = cl.KvBatch(torch.tensor(lens, dtype=torch.int32).cuda(), p.table.cuda(), N + 9, q_len=max(counts), q_start=start,
                           max_kv_len=int(max(lens)), prefix_table=pre, prefix_len=prefix)
        q, k, v = (torch.from_numpy(g.standard_normal((N + 9, h, D)) * 2.0 ** g.integers(-4, 5, (N + 9, 1, 1))).to(dtype) for h in (5, Hkv, Hkv))
        out = torch.full_like(q, 7.0).cuda()
        cl.kv_append(p.cache, batch, k.cuda(), v.cuda(), q=q.cuda(), rope=rope, q_norm=w.cuda() if norm else None,
                     k_norm=w.cuda() if norm else None, q_out=out)
        torch.cuda.synchronize()
        wd, mine = (w.double().numpy() if norm else None), slice(ahead, ahead + N)
        p.check(lens, counts, turned(k[mine].double().numpy(), lens, counts, freq.double().numpy(), inter, wd), v[mine].double().numpy())
        ref = turned(q[mine].double().numpy(), lens, counts, freq.double().numpy(), inter, wd)
        far = np.abs(ref).max(axis=-1, keepdims=True)
        u = 2.0 ** (-11 if dtype == F16 else -8)
        assert (np.abs(out[mine].double().cpu().numpy() - ref) <= u * np.abs(ref) * 1.01 + 2.0 ** -20 * far + 2.0 ** -25).all()
        assert (out[:ahead] == 7).all() and (out[ahead + N:] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
def test_append_without_rotation_or_queries(dtype):
    """V's path for K too: codes equal the oracle's bit for bit, in prompts and in single tokens."""
    g = torch.Generator().manual_seed(9)
    for counts in ([600, 100], [1, 1]):
        p = Pool([700, 300], 2, 128, 32, 32, dtype)
        k, v = (torch.randn((sum(counts), 2, 128), generator=g).to(dtype) for _ in range(2))
        assert cl.kv_append(p.cache, p.batch([690, 111], counts), k.cuda(), v.cuda()) is None
        torch.cuda.synchronize()
        p.check([690, 111], counts, k.double().numpy(), v.double().numpy(), rel=0.0)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
def test_append_ends_of_the_range(dtype):
    """Zeros, the type's largest and smallest values, infinities, NaN, and blocks that grow from one end to the other."""
    p = Pool([64], 2, 64, 32, 16, dtype)
    big = torch.finfo(dtype).max
    rows = torch.zeros((20, 2, 64), dtype=dtype)
    rows[1] = torch.finfo(dtype).smallest_normal
    rows[2, :, ::2] = torch.finfo(dtype).smallest_normal * 2.0 ** -6
    rows[3], rows[4, :, 5] = 1.0, big
    rows[5, 0, 1], rows[5, 1, 2], rows[6, 0, 0] = float("inf"), float("-inf"), float("nan")
    rows[7], rows[17] = -big, 3.0
    at = 0
    for a in (1, 1, 1, 1, 1, 2, 1, 9, 3):
        new = rows[at:at + a]
        at += a
        cl.kv_append(p.cache, p.batch([at], [a]), new.cuda(), new.cuda())
        torch.cuda.synchronize()
        p.check([at], [a], new.double().numpy(), new.double().numpy(), rel=0.0)
    k, v = cl.kv_read(p.cache, p.batch([20], [20]))
    assert torch.equal(k.nan_to_num(9.0), v.nan_to_num(9.0)) and not k.isinf().any()
    assert torch.equal(k.cpu().isnan(), ~rows.isfinite())


def test_append_leaves_shared_and_missing_pages_alone():
    g = torch.Generator().manual_seed(4)
    p = Pool([70, 50, 10], 2, 64, 16, 8, F16, prefix=20)
    p.table[1, 1] = -1
    p.table[0, 2] = 1 << 30
    lens, counts = [70, 50, 10], [55, 41, 10]                     # below the prefix, and wholly inside it
    N = sum(counts)
    k, v = (torch.randn((N, 2, 64), generator=g).half() for _ in range(2))
    cl.kv_append(p.cache, p.batch(lens, counts), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    p.check(lens, counts, k.double().numpy(), v.double().numpy(), rel=0.0)


def test_append_of_views_and_positions():
    """k, v and q as unaligned views of a fused projection, angles from given positions."""
    g = torch.Generator().manual_seed(5)
    D, Hq, Hkv, N = 64, 4, 2, 21
    wide = torch.randn((N, 1 + (Hq + 2 * Hkv) * D), generator=g).to(BF16).cuda()
    parts = wide[:, 1:].split([Hq * D, Hkv * D, Hkv * D], 1)
    q, k, v = (x.unflatten(1, (-1, D)) for x in parts)
    freq = cl.rope_frequencies(D, 10000.0)[0]
    pos = torch.arange(N, dtype=torch.int32).cuda() * 3 + 1000
    out, pools = [], []
    for a, b, c in ((q, k, v), tuple(x.contiguous() for x in (q, k, v))):
        p = Pool([40], Hkv, D, 16, 16, BF16)
        out.append(cl.kv_append(p.cache, p.batch([40], [N]), b, c, q=a, rope=cl.Rope(freq.cuda()), positions=pos))
        pools.append(p)
    torch.cuda.synchronize()
    assert torch.equal(*out) and torch.equal(pools[0].cache.k, pools[1].cache.k)
    x = k.double().cpu().numpy()
    ref = np.stack([layer.rotate(x[i], int(pos[i]), freq.double().numpy()) for i in range(N)])
    pools[0].check([40], [N], ref, v.double().cpu().numpy())


def test_rows_of_no_sequence_are_left_alone():
    p = Pool([40, 50], 2, 64, 16, 16, F16)
    start = torch.tensor([1, 3, 6], dtype=torch.int32, device="cuda")
    b = cl.KvBatch(torch.tensor([40, 50], dtype=torch.int32, device="cuda"), p.table.cuda(), 8, q_len=3, q_start=start, max_kv_len=50)
    x = torch.randn((8, 2, 64), device="cuda").half()
    q = torch.full((8, 2, 64), 7.0, device="cuda").half()
    cl.kv_append(p.cache, b, x, x, q=x, q_out=q)
    k, v = (torch.full((8, 2, 64), 7.0, device="cuda").half() for _ in range(2))
    cl.kv_read(p.cache, b, k=k, v=v)
    torch.cuda.synchronize()
    for y in (q, k, v):
        assert (y[0] == 7).all() and (y[6:] == 7).all()
    assert torch.equal(q[1:6], x[1:6]) and ((v[1:6] - x[1:6]).abs() <= 2.0 ** -4 * x[1:6].abs() + 2.0 ** -9).all()


@pytest.mark.parametrize("eight", [False, True], ids=["16bit", "8bit"])
@pytest.mark.parametrize("D,Hkv", [(128, 3), (64, 1), (256, 2)])
def test_read_of_whole_sequences(D, Hkv, eight):
    """More rows than a call takes a workgroup each: sequences from their first key on, one asked for more rows than it has
    keys, pages outside the pool, rows of no sequence on both sides."""
    lens, page, ahead = [1500, 700, 30, 1], 16, 3
    p = Pool(lens, Hkv, D, page, 8, BF16)
    if eight:
        cache, val = p.cache, [decoded(p.t[i], p.t[2 + i], 8, BF16) for i in (0, 1)]
    else:
        val = [torch.randn(p.t[0].shape).to(BF16) for _ in range(2)]
        cache = cl.KvCache(*[v.cuda() for v in val])
    p.table[1, 2] = len(p.t[0])
    counts = [1500, 700, 35, 1]
    start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + ahead, dtype=torch.int32).cuda()
    N = sum(counts) + 2 * ahead + 1
    batch = cl.KvBatch(torch.tensor(lens, dtype=torch.int32).cuda(), p.table.cuda(), N, q_len=1500, q_start=start, max_kv_len=1500)
    out = [torch.full((N, Hkv, D), 7.0, device="cuda").to(BF16) for _ in range(2)]
    cl.kv_read(cache, batch, *out)
    torch.cuda.synchronize()
    for got, v in zip(out, val):
        got = got.cpu()
        assert (got[:ahead] == 7).all() and (got[N - ahead - 1:] == 7).all()
        at = ahead
        for b, (n, a) in enumerate(zip(lens, counts)):
            for i in range(a):
                j = n - a + i
                row = got[at + i]
                if j < 0:
                    assert (row == 0).all()
                elif b == 1 and j // page == 2:
                    assert row.isnan().all()
                else:
                    assert torch.equal(row, v[int(p.table[b, j // page]), :, j % page])
            at += a


def test_read_of_a_16_bit_cache():
    c = Case([3, 2], [40, 30], 4, 2, 64, 16, BF16, prefix=10)
    k, v = cl.kv_read(c.cache, c.batch)
    torch.cuda.synchronize()
    at = 0
    for b, (a, n) in enumerate(zip(c.q_lens, c.kv_lens)):
        for got, ref in ((k, c.ks[b]), (v, c.vs[b])):
            assert np.array_equal(got[at:at + a].double().cpu().numpy(), ref[:, n - a:].transpose(1, 0, 2))
        at += a
    # positions below 0, the prefix, and a page outside the pool
    c.table[0, 1] = -1
    start = torch.tensor([0, 45, 50], dtype=torch.int32, device="cuda")
    k, _ = cl.kv_read(c.cache, cl.KvBatch(c.batch.kv_len, c.table, 50, q_len=45, q_start=start, max_kv_len=40,
                                          prefix_table=c.batch.prefix_table, prefix_len=10))
    k = k.double().cpu().numpy()
    assert (k[:5] == 0).all() and np.array_equal(k[5:31], c.ks[0][:, :26].transpose(1, 0, 2)) and np.isnan(k[31:45]).all()


def test_a_stream_of_its_own_beside_a_busy_one():
    """Calls on another stream take their workspaces and results there: memory that queued work still reads is not theirs."""
    c = Case8([1, 2, 1], [5000, 3000, 4000], 8, 2, 128, 16, F16)
    q = c.q.cuda()
    want = cl.attention(c.cache, c.batch, q, out_dtype=F32)
    kept = cl.kv_read(c.cache, c.batch)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.ones((4096, 4096), device="cuda")
    for _ in range(4):
        x = torch.full((cl.attention_workspace(c.cache, c.batch, 8) // 4,), 3.0, device="cuda")
        for _ in range(20):
            big = (big @ big).clamp_(max=1.0)
        keep = x * 2
        del x
        got = cl.attention(c.cache, c.batch, q, out_dtype=F32, stream=side)
        read = cl.kv_read(c.cache, c.batch, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool((keep == 6.0).all()) and all(torch.equal(a, b) for a, b in zip(read, kept))


def test_results_repeat_on_other_streams_and_in_graphs():
    """Append, read and attention as one captured step, replayed with eager work between."""
    c = Case8([1] * 6, [5000, 3000, 400, 17, 16, 900], 8, 2, 128, 16, BF16, block=16, spare=0)
    pools = [[x.clone() for x in (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale)] for _ in range(2)]
    caches = [cl.KvCache8(*x, BF16) for x in pools]
    k, v = (torch.randn((6, 2, 128), device="cuda").to(BF16) for _ in range(2))
    q = c.q.cuda()

    def step(cache):
        cl.kv_append(cache, c.batch, k, v)
        return (cl.attention(cache, c.batch, q), *cl.kv_read(cache, c.batch))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in caches:
            step(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0])
    for i in range(4):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, device="cuda") * (i + 1))
        want = step(caches[1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(*pools))
