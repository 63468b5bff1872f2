"""Beam search through all of its calls (reserve, append, attention, select, fork, gather, free) over caches of 16 and 8 bits:
every hypothesis' score is that of its tokens run as one prompt over a cache of its own, the best first step is the
oracle's, and the pool is left as it was found."""

import numpy as np
import pytest
import torch

from oracle import beam
from paper_2605_05819_amd import cl, decoder
from tests.test_decoder_gpu import D, HIDDEN, HKV, Layer

pytestmark = pytest.mark.gpu

VOCAB, PAGE = 61, 8


def model(eight, pages, layers=2):
    stack = [Layer(False, 1, seed=i) for i in range(layers)]
    norms = [s.norms[0] for s in stack] + [stack[0].norms[2]]
    make = (lambda: cl.KvCache8.empty(pages, PAGE, HKV, D, 4)) if eight else (lambda: cl.KvCache.empty(pages, PAGE, HKV, D))
    caches = [make() for _ in stack]
    g = torch.Generator(device="cuda").manual_seed(8)
    embed = torch.randn((VOCAB, HIDDEN), device="cuda", generator=g).half()
    head = (torch.randn((VOCAB, HIDDEN), device="cuda", generator=g) * 0.15).half()
    pool = cl.PagePool.of(caches, torch.zeros(1, dtype=torch.int32, device="cuda"))
    return [s.dev for s in stack], norms, caches, pool, embed, head


def log_probs(m, tokens):
    """[tokens][VOCAB] of one sequence as a prompt, fp64, over fresh pages of the same kind of cache."""
    layers, norms, caches, _, embed, head = m
    fresh = [type(c).empty(-(-len(tokens) // PAGE), PAGE, HKV, D, *([c.block] if isinstance(c, cl.KvCache8) else [])) for c in caches]
    n = len(tokens)
    batch = cl.KvBatch(torch.tensor([n], dtype=torch.int32, device="cuda"), torch.arange(-(-n // PAGE), dtype=torch.int32, device="cuda")[None],
                       n, q_len=n, max_kv_len=n)
    _, y = decoder.run(layers, fresh, batch, embed[tokens.long()], norms[:-1], norms[-1])
    return torch.log_softmax(torch.mm(y, head.t(), out_dtype=torch.float32).double(), 1).cpu().numpy()


@pytest.mark.parametrize("eight", [False, True], ids=["16bit", "8bit"])
@pytest.mark.parametrize("eos,alpha", [(-1, 0.0), (7, 0.6)])
def test_hypotheses_score_as_their_tokens(eight, eos, alpha):
    """Steps of a few tokens come by the decode calls, the whole sequence by one prompt: fp16 roundings between the calls
    differ (1e-2 of the norms in all, as for the layer's own test), which moves a log probability of 12 tokens by less
    than 12 x 2 x 1e-2 x the logits' size (3 or so)."""
    m = model(eight, 60)
    layers, norms, caches, pool, embed, head = m
    prompts = [torch.tensor(p, dtype=torch.int32, device="cuda") for p in ([3, 1, 4, 1, 5, 9, 2, 6, 5], [11], [20] * 16)]
    steps, beams = 12, 4
    rule = cl.Beams(beams, eos=eos, alpha=alpha)
    got = decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head, prompts, rule, steps)
    torch.cuda.synchronize()
    assert int(pool.refs.abs().sum()) == 0 and int(pool.missing) == 0
    size = got.lengths.cpu().numpy()
    for r in range(beams * len(prompts)):
        p, t = prompts[r // beams], got.tokens[r, :size[r]]
        assert bool(got.finished[r]) == (eos in t.tolist()) and (bool(got.finished[r]) or size[r] == steps)
        lp = log_probs(m, torch.cat([p, t[:-1]]))[len(p) - 1:]
        want = lp[np.arange(size[r]), t.cpu().numpy()].sum()
        assert abs(float(got.scores[r]) - want) <= 0.7, (r, float(got.scores[r]), want)
    rank = (got.scores.double().cpu().numpy() / np.maximum(size, 1) ** alpha).reshape(-1, beams)
    assert (np.diff(rank, axis=1) <= 1e-6).all()
    rows = [tuple(x) for x in got.tokens.tolist()]
    assert len({(i // beams, x) for i, x in enumerate(rows)}) == len(rows)          # no hypothesis twice


def test_one_step_is_the_best_tokens():
    m = model(True, 20)
    layers, norms, caches, pool, embed, head = m
    p = torch.tensor([3, 1, 4, 1, 5], dtype=torch.int32, device="cuda")
    got = decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head, [p], cl.Beams(5), 1)
    lp = log_probs(m, p)[-1:]
    s, t, _, _, _, _ = beam.select(lp, [0.0], 1, 5)
    assert got.tokens[:, 0].tolist() == t[0].astype(int).tolist() and np.allclose(got.scores.cpu().numpy(), s[0], atol=1e-5)


def test_a_full_pool_is_an_error():
    m = model(True, 6)
    layers, norms, caches, pool, embed, head = m
    p = torch.arange(30, dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError, match="pages too few"):
        decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head, [p], cl.Beams(4), 12)
    assert int(pool.refs.abs().sum()) == 0


def test_refusals():
    m = model(False, 6)
    layers, norms, caches, pool, embed, head = m
    call = lambda rule, pool=pool, n=1: decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head,  # noqa: E731
                                                            [torch.zeros(1, dtype=torch.int32, device="cuda")] * n, rule, 1)
    with pytest.raises(ValueError, match="picks"):
        call(cl.Beams(2, picks=4))
    with pytest.raises(ValueError, match="rows"):
        call(cl.Beams(33), n=2)
    with pytest.raises(ValueError, match="missing"):
        call(cl.Beams(2), cl.PagePool.of(caches))
    with pytest.raises(ValueError, match="at least one token"):
        call(cl.Beams(2), n=0)
    with pytest.raises(ValueError, match="at least one token"):
        decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head,
                            [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (3, 0)], cl.Beams(2), 1)


def test_the_example_runs(capsys):
    decoder.main(layers=1, seqs=2, prompt=70, steps=4, page=16)
    out = capsys.readouterr().out
    assert "prompt:" in out and "decode:" in out and "beam search: 4 x 4" in out
