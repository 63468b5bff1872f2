"""How a beam search leaves its pool: every page given back, whatever ends it, and its count of missing pages added to."""

import pytest
import torch

from paper_2605_05819_amd import cl, decoder
from tests.test_beam_search_gpu import PAGE, model
from tests.test_decoder_gpu import D, HKV, Layer

pytestmark = pytest.mark.gpu


def search(m, prompts, beams=3, steps=6):
    layers, norms, caches, pool, embed, head = m
    return decoder.beam_search(layers, caches, pool, norms[:-1], norms[-1], embed, head,
                               [torch.tensor(p, dtype=torch.int32, device="cuda") for p in prompts], cl.Beams(beams), steps)


def held(pool):
    torch.cuda.synchronize()
    return int(pool.refs.abs().sum())


@pytest.mark.parametrize("call", [1, 2, 3, 6])
def test_pages_are_given_back_when_a_step_fails(call, monkeypatch):
    """A failure in the prompts' step and in later ones, ahead of the search's end; the next search finds the whole pool."""
    m = model(True, 30)
    prompts = [[3, 1, 4, 1, 5, 9, 2, 6, 5], [11]]
    want = search(m, prompts)
    calls, whole = [0], decoder.run

    def run(*args):
        calls[0] += 1
        if calls[0] == call:
            raise MemoryError("none left")
        return whole(*args)

    with monkeypatch.context() as patch:
        patch.setattr(decoder, "run", run)
        with pytest.raises(MemoryError):
            search(m, prompts)
    assert held(m[3]) == 0
    got = search(m, prompts)
    assert torch.equal(got.tokens, want.tokens) and torch.equal(got.scores, want.scores) and held(m[3]) == 0


def test_prompts_too_long_for_experts():
    """65 tokens behind the reservation of their pages: the layer of experts refuses them."""
    layers, norms, caches, pool, embed, head = model(False, 30)
    moe = Layer(True, 1)
    caches = [cl.KvCache.empty(30, PAGE, HKV, D)]
    pool = cl.PagePool.of(caches, torch.zeros(1, dtype=torch.int32, device="cuda"))
    m = [moe.dev], [moe.norms[0], moe.norms[2]], caches, pool, embed, head
    with pytest.raises(ValueError, match="64 tokens"):
        search(m, [list(range(40)), [5] * 25])
    assert held(pool) == 0
    assert search(m, [list(range(40)), [5] * 24]).tokens.shape == (6, 6) and held(pool) == 0


def test_the_count_of_missing_pages_goes_on():
    """What earlier calls lacked is neither an error of this search nor lost; what this one lacks is added."""
    m = model(False, 6)
    pool = m[3]
    table, n = torch.full((1, 9), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cl.kv_reserve(pool, table, n, torch.full_like(n, 9 * PAGE))       # 9 pages of 6
    assert int(pool.missing) == 3
    cl.kv_free(pool, table, n)
    search(m, [[3, 1, 4]], beams=2, steps=3)
    assert int(pool.missing) == 3 and held(pool) == 0
    with pytest.raises(RuntimeError, match="pages too few") as e:
        search(m, [list(range(30))], beams=4, steps=12)
    assert int(pool.missing) == 3 + int(str(e.value).split("had ")[1].split()[0]) and held(pool) == 0
    search(m, [[3, 1, 4]], beams=2, steps=3)
