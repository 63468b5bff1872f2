"""Every hypothesis of a beam search against the same calls without any sharing: the prompts' step over the same batch, then
each row's own tokens one by one, over pages that are only its own and hold what the prompts' step left (copied by
torch).  The calls, their batch sizes and the places of blocks and pages in a sequence are the same, and a row's result
depends on its own data alone, so the logits of each step are those of the search bit for bit.  Left are the sums: a
score is rounded to fp32 at each step (half a step of 2^-18 at scores of up to 64: 2^-19), and a step's log-sum is
off by 2^-21 at most, in 12 steps 12 (2^-19 + 2^-21) < 2^-15."""

import numpy as np
import pytest
import torch

from paper_2605_05819_amd import cl, decoder
from tests.test_beam_search_gpu import PAGE, model
from tests.test_decoder_gpu import D, HKV

pytestmark = pytest.mark.gpu


def fresh(cache, pages):
    """A cache of the same kind and number of pages, its bytes zero."""
    if isinstance(cache, cl.KvCache8):
        new = cl.KvCache8.empty(pages, PAGE, HKV, D, cache.block)
        parts = new.k, new.v, new.k_scale, new.v_scale
    else:
        new = cl.KvCache.empty(pages, PAGE, HKV, D)
        parts = new.k, new.v
    for x in parts:
        x.zero_()
    return new, parts


def replay(m, prompts, tokens, beams):
    """log probabilities fp64 [rows][steps][vocab] of rows that feed ``tokens`` behind their prompts."""
    layers, norms, caches, _, embed, head = m
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rows, steps = tokens.shape
    counts = [len(p) for p in prompts]
    width = -(-(max(counts) + steps) // PAGE)
    mine = [fresh(c, (len(prompts) + rows) * width) for c in caches]
    own = [x[0] for x in mine]
    table = torch.arange((len(prompts) + rows) * width, dtype=torch.int32, device="cuda").view(-1, width)
    start = i32(np.concatenate([[0], np.cumsum(counts)]).tolist())
    batch = cl.KvBatch(i32(counts), table[:len(prompts)].contiguous(), sum(counts), q_len=max(counts), q_start=start,
                       max_kv_len=max(counts))
    _, y = decoder.run(layers, own, batch, embed[torch.cat(prompts).long()], norms[:-1], norms[-1])
    for _, parts in mine:
        for x in parts:
            x[table[len(prompts):].long()] = x[table[:len(prompts)].long()].repeat_interleave(beams, 0)
    out = [torch.mm(y[(start[1:] - 1).long()], head.t(), out_dtype=torch.float32).repeat_interleave(beams, 0)]
    kv_len = i32(counts).repeat_interleave(beams)
    for step in range(steps - 1):
        kv_len = kv_len + 1
        batch = cl.KvBatch(kv_len, table[len(prompts):].contiguous(), rows, max_kv_len=max(counts) + step + 1)
        _, y = decoder.run(layers, own, batch, embed[tokens[:, step].long()], norms[:-1], norms[-1])
        out.append(torch.mm(y, head.t(), out_dtype=torch.float32))
    return torch.log_softmax(torch.stack(out, 1).double(), 2).cpu().numpy()


@pytest.mark.parametrize("eight", [False, True], ids=["16bit", "8bit"])
@pytest.mark.parametrize("eos,alpha", [(-1, 0.0), (7, 0.6)])
def test_hypotheses_score_as_their_tokens_over_unshared_pages(eight, eos, alpha):
    m = model(eight, 60)
    layers, norms, caches, pool, embed, head = m
    prompts = [torch.tensor(p, dtype=torch.int32, device="cuda") for p in ([3, 1, 4, 1, 5, 9, 2, 6, 5], [11], [20] * 16)]
    steps, beams = 12, 4
    got = decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head, prompts,
                              cl.Beams(beams, eos=eos, alpha=alpha), steps)
    lp = replay(m, prompts, got.tokens, beams)
    torch.cuda.synchronize()
    size, tokens, scores = got.lengths.tolist(), got.tokens.tolist(), got.scores.double().tolist()
    assert max(abs(s) for s in scores) < 64
    for r, (n, t, s) in enumerate(zip(size, tokens, scores)):
        want = sum(lp[r, i, t[i]] for i in range(n))
        assert abs(s - want) <= 2.0 ** -15, (r, s, want)
    # the rows did go over each other's pages: hypotheses of a prompt share their first tokens
    assert any(tokens[r][:3] == tokens[r + 1][:3] for r in range(len(tokens) - 1) if (r + 1) % beams)
