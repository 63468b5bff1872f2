"""Prompts beside single tokens over a cache of 8 bits: each sequence's keys are converted ahead, or not, by its own new
tokens, and the workspace holds those that can be long."""

import ctypes

import pytest
import torch

from paper_2605_05819_amd import cl

FAKE = 0x100000


def workspace(q_heads=32, kv_heads=8, dim=128, page=16, q_start=FAKE, **kw):
    pages = 0x7fffffff // (kv_heads * page)
    c = cl.KvCache8C(FAKE, FAKE, FAKE, FAKE, pages, page, kv_heads, dim, page, cl.CL_BF16)
    b = cl.KvBatchC(q_start, FAKE, FAKE, 0, kw["seqs"], kw["tokens"], kw["q_len"], -(-kw["keys"] // page), 0, kw["keys"])
    c2 = cl.KvCacheC(FAKE, FAKE, pages, page, kv_heads, dim, cl.CL_BF16)
    lib = cl.lib()
    return (lib.cl_attention8_workspace(ctypes.byref(c), ctypes.byref(b), q_heads) -
            lib.cl_attention_workspace(ctypes.byref(c2), ctypes.byref(b), q_heads))


def test_the_workspace_is_that_of_the_long_sequences():
    key = 2 * 8 * 128 * 2                                 # a key and its value in 16 bits, bytes
    # 1000 tokens beside 15 single ones: sequences of 8 blocks of 128 rows and more, four at most of 1015 tokens
    got = workspace(seqs=16, tokens=1015, q_len=1000, keys=8192)
    assert 8192 * key <= got <= 4 * 8192 * key + 4 * 4 * 512 + 1024
    # sequences of one length are all of them long
    assert workspace(seqs=4, tokens=4000, q_len=1000, keys=8192, q_start=0) >= 4 * 8192 * key
    assert workspace(seqs=4, tokens=4000, q_len=1000, keys=8192) >= 4 * 8192 * key
    # 300 single tokens do not keep a prompt's keys from being converted
    got = workspace(seqs=301, tokens=2300, q_len=2000, keys=8192)
    assert 8192 * key <= got <= 11 * 8192 * key + 11 * 4 * 512 + 4 * 301 + 1024
    # nothing is, for a few tokens each or past 1 GiB of keys
    assert workspace(seqs=16, tokens=64, q_len=4, keys=8192) == 0
    assert workspace(seqs=1, tokens=2000, q_len=2000, keys=1 << 20) == 0


SHAPES = [
    ([520, 1, 1, 4, 1], [700, 900, 1, 333, 64], 16, 4, 128, 16, 16),
    ([1, 1, 530, 0, 1, 260, 2], [640, 31, 530, 50, 0, 300, 70], 16, 4, 64, 64, 8),
    ([3, 300, 1, 150, 40], [515, 400, 333, 150, 41], 16, 4, 256, 32, 32),
    ([255, 256, 257, 1, 512], [255, 300, 400, 200, 600], 16, 4, 128, 16, 1),         # on both sides of 8 blocks of 128 rows
    ([1] * 70 + [600] + [1] * 70 + [300], [5 + i for i in range(70)] + [800] + [90 - i for i in range(70)] + [310], 8, 2, 64, 16, 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_oracle(shape, dtype):
    from tests.test_cache8_gpu import Case8, check
    q, kv, Hq, Hkv, D, page, block = SHAPES[shape]
    c = Case8(q, kv, Hq, Hkv, D, page, dtype, block=block, seed=shape)
    assert cl.attention_workspace(c.cache, c.batch, Hq) >= max(kv) * 4 * Hkv * D
    check(c)
    check(c, causal=False, window=(0, 70, 1, 130, 33)[shape], out_dtype=torch.float32)


@pytest.mark.gpu
def test_only_long_sequences_are_converted():
    """Of a workspace of 255s, what the call writes: two sequences' keys and values, their pages and places."""
    from tests.test_cache8_gpu import Case8
    q, kv, Hq, Hkv, D, page = [600, 1, 1, 310, 5, 1], [768, 1024, 1000, 512, 64, 3], 16, 4, 128, 16
    c = Case8(q, kv, Hq, Hkv, D, page, torch.float16, block=16, seed=1)
    x = c.q.cuda()
    need = cl.attention_workspace(c.cache, c.batch, Hq)
    split = cl.attention_workspace(c.twin, c.batch, Hq)               # of a 16-bit cache: the splits' part
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out = cl.attention(c.cache, c.batch, x, ws=ws)
    torch.cuda.synchronize()
    # more than 7 blocks of 128 rows are 225 tokens of 4 heads: of 918 tokens 4 sequences at most
    keys, slots, pages = 768 + 512, 918 // 225, 1024 // page
    pool = ws[split:].view(torch.int32)[:2 * slots * 1024 * Hkv * D // 2]
    assert abs(int((pool != -1).sum()) - keys * Hkv * D) <= 2        # 16-bit pairs of codes that happen to be 0xffff 0xffff: NaN, none here
    table = ws[split + 4 * slots * 1024 * Hkv * D:].view(torch.int32)[:slots * pages].view(slots, pages)
    assert (table[0, :48] == torch.arange(48, device="cuda")).all() and (table[0, 48:] == -1).all()
    assert (table[1, :32] == pages + torch.arange(32, device="cuda")).all() and (table[1, 32:] == -1).all() and (table[2:] == -1).all()
    want = cl.attention(c.twin, c.batch, x)
    torch.cuda.synchronize()
    assert torch.equal(out[:600], want[:600]) and torch.equal(out[602:912], want[602:912])


@pytest.mark.gpu
def test_a_graph_whose_sequences_change_places():
    """One captured call, replayed while starts and lengths move: which sequences are long is the device's to see."""
    from tests.test_cache8_gpu import Case8
    Hq, Hkv, D, page = 16, 4, 128, 16
    c = Case8([520, 1, 1, 300], [640, 640, 640, 640], Hq, Hkv, D, page, torch.float16, block=16, seed=2)
    x, out = c.q.cuda(), torch.empty_like(c.q, device="cuda")
    ws = torch.full((cl.attention_workspace(c.cache, c.batch, Hq),), 255, dtype=torch.uint8, device="cuda")
    start, lens = c.batch.q_start, c.batch.kv_len
    run = lambda: cl.attention(c.cache, c.batch, x, out=out, ws=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for q, kv in (([520, 1, 1, 300], [640] * 4), ([1, 300, 520, 1], [640, 512, 600, 33]), ([2, 1, 1, 1], [640, 2, 1, 64]),
                  ([0, 224, 225, 373], [5, 640, 640, 640]), ([520, 302, 0, 0], [640, 640, 640, 0])):
        s = [0]
        for n in q:
            s.append(s[-1] + n)
        start.copy_(i32(s)), lens.copy_(i32(kv))
        want = cl.attention(c.twin, c.batch, x)                # of the 16-bit cache of the same values
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[s[-1]:], torch.full_like(out[s[-1]:], 7.0))
        # two results' outputs and probabilities, each rounded by 2^-11 at most: 2^-9
        off = (out[:s[-1]].float() - want[:s[-1]].float()).abs()
        assert (off <= 2.0 ** -9 * want[:s[-1]].float().abs() + 2.0 ** -12).all()
        eager = cl.attention(c.cache, c.batch, x)
        torch.cuda.synchronize()
        assert torch.equal(out[:s[-1]], eager[:s[-1]])
