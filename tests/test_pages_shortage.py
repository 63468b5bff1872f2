"""Pools that run out, and last pages whose holders all grow: no row loses keys that it held, a call that is made again
gets what was missing, and a page stays with one of its holders where all of them would leave it."""

import random

import pytest
import torch

from oracle import pages


def test_all_holders_grow_and_the_first_keeps_the_page():
    # rows 0 and 1 share page 1 (6 keys of pages of 4); one page is free
    refs, table = [2, 2, 0], [[0, 1, -1], [0, 1, -1]]
    copies, missing = pages.reserve(refs, table, [6, 6], [7, 7], 4)
    assert copies == [(1, 2)] and missing == 0 and table == [[0, 1, -1], [0, 2, -1]] and refs == [2, 1, 1]
    # a holder that does not grow keeps it: the other one copies
    refs, table = [2, 2, 0], [[0, 1, -1], [0, 1, -1]]
    copies, missing = pages.reserve(refs, table, [6, 6], [7, 6], 4)
    assert copies == [(1, 2)] and missing == 0 and table == [[0, 2, -1], [0, 1, -1]] and refs == [2, 1, 1]


def test_a_row_without_a_page_for_its_copy_keeps_the_shared_one():
    # rows 0, 1 and 2 share page 1, row 3 has page 2: no page is free
    refs, table, lens = [3, 3, 1], [[0, 1, -1], [0, 1, -1], [0, 1, -1], [2, -1, -1]], [6, 6, 6, 4]
    copies, missing = pages.reserve(refs, table, lens, [7, 7, 6, 4], 4)
    assert copies == [] and missing == 2 and table == [[0, 1, -1]] * 3 + [[2, -1, -1]] and refs == [3, 3, 1]
    # row 3 ends: of the two that ask again the first gets its page
    pages.free(refs, table, lens, [3])
    copies, missing = pages.reserve(refs, table, lens, [7, 7, 6, 0], 4)
    assert copies == [(1, 2)] and missing == 1 and table[:3] == [[0, 2, -1], [0, 1, -1], [0, 1, -1]] and refs == [3, 2, 1]


def test_children_of_different_parents():
    # rows 0 and 1 share page 0 and have two children and one
    refs, table = [2, 0, 0], [[0, -1], [0, -1]]
    new, n, copies, missing = pages.fork(refs, table, [3, 3], [1, 0, 0], 4, room=1)
    assert new == [[0, -1], [1, -1], [2, -1]] and copies == [(0, 1), (0, 2)] and missing == 0 and refs == [1, 1, 1]


def _rows(w):
    """The bytes of every row's keys, by its table."""
    out, bufs = [], [x.cpu() for x in w.buffers()]
    for t, n in zip(w.table.tolist(), w.len.tolist()):
        own = max(n - w.prefix, 0)
        keys = []
        for j in range(own):
            page = t[j // w.size]
            # a page is [heads][rows] of bytes: those of row j % size of each head
            for b, heads in zip(bufs, w.heads):
                per = b.shape[1] // heads
                one = per // w.size if per % w.size == 0 and per >= w.size else 0
                if one:
                    x = b[page].view(heads, w.size, one)[:, j % w.size]
                    keys.append(bytes(x.contiguous().numpy()))
        out.append(keys)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(16))
def test_scarce_pools_lose_no_keys(seed):
    """Forks without room, so that last pages are shared by rows of several parents, then forks and reservations over a
    pool with few free pages: equal to the oracle, and every row's keys what they were."""
    from tests.test_pages_gpu import World
    g = random.Random(seed)
    size, heads = g.choice((4, 16)), 2
    w = World(g.randint(12, 40), size, g.randint(2, 6), g.randint(2, 7), layers=g.randint(1, 2), heads=heads, eight=seed % 2 == 1,
              prefix=g.choice((0, 0, 3)), seed=seed)
    w.heads = [heads] * len(w.buffers())
    w.reserve([g.randint(0, 3 * size) for _ in w.n])
    w.set([w.prefix + min(g.randint(1, 3 * size), size * sum(p >= 0 for p in t)) if t[0] >= 0 else 0 for t in w.t])
    w.check()
    for _ in range(10):
        parents = [g.randint(0, len(w.t) - 1) for _ in range(g.randint(1, 24))]
        before = _rows(w)
        room = g.choice((0, 0, 1, size + 1))
        w.fork(parents, room)
        w.check()
        assert _rows(w) == [before[p] for p in parents]
        before = _rows(w)
        want = [x + g.choice((0, 1, 1, size)) for x in w.n]
        w.reserve(want)
        w.check()
        assert _rows(w) == before
        if w.short and g.random() < 0.5:              # give some back and ask again
            w.free([g.randint(0, len(w.t) - 1) for _ in range(3)])
            before = _rows(w)
            w.reserve([max(a, b) if b else 0 for a, b in zip(want, w.n)])
            w.check()
            assert _rows(w) == before


@pytest.mark.gpu
def test_many_rows_share_and_grow():
    """More rows than the scanning workgroup has threads, groups of them over one last page each."""
    from tests.test_pages_gpu import World
    g = random.Random(5)
    w = World(1600, 4, 300, 3, layers=1, heads=1, seed=1)
    w.reserve([6] * 300)
    w.set([6] * 300)
    w.fork([g.randint(0, 299) for _ in range(1500)], 0)
    w.check()
    w.reserve([x + (g.random() < 0.9) for x in w.n])
    w.check()
    w.fork(list(range(1500)), 1)
    w.check()
