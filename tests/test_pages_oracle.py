"""Pins of the oracles of pages and beams: worked by hand, and what has to hold for any calls."""

import random

import numpy as np

from oracle import beam, pages


def test_fork_by_hand():
    # pages of 4 keys: row 0 has 6 keys on pages 2, 5; row 1 8 keys on 0, 1 and page 3 ahead; 4 and 6 are free
    refs, table, lens = [1, 1, 1, 1, 0, 1, 0], [[2, 5, -1], [0, 1, 3]], [6, 8]
    new, n, copies, missing = pages.fork(refs, table, lens, [0, 1, 0, -1], 4, room=1)
    # the first child of 0 keeps page 5, the second copies it to 4; row 1's child keeps page 3 ahead
    assert new == [[2, 5, -1], [0, 1, 3], [2, 4, -1], [-1, -1, -1]] and n == [6, 8, 6, 0]
    # (row 1's next key is page 3's), the row without a parent gets nothing
    assert copies == [(5, 4)] and missing == 0 and refs == [1, 1, 2, 1, 1, 1, 0]


def test_fork_by_hand_empty_rows_take_pages():
    refs = [0, 0, 0]
    new, n, copies, missing = pages.fork(refs, [[-1, -1]], [0], [0, 0], 4, room=5)
    assert new == [[0, 1], [2, -1]] and n == [0, 0] and copies == [] and missing == 1 and refs == [1, 1, 1]


def test_compact_by_hand():
    refs, t = [0, 2, 0, 1, 1, 0], [4, 1, -1, 3, 1, 5]
    assert pages.compact(refs, [t]) == [(3, 0), (4, 2)]
    assert refs == [1, 2, 1, 0, 0, 0] and t == [2, 1, -1, 0, 1, -1]


def test_counts_are_the_holders_whatever_is_called():
    g = random.Random(1)
    for _ in range(200):
        num, size, rows, width = g.randint(3, 40), g.choice((1, 4, 16)), g.randint(1, 6), g.randint(1, 8)
        refs, table, lens = [0] * num, [[-1] * width for _ in range(rows)], [0] * rows
        content = {}
        for _ in range(12):
            what = g.choice(("reserve", "fork", "free", "compact"))
            if what == "reserve":
                want = [x + g.randint(0, 2 * size) for x in lens]
                copies, _ = pages.reserve(refs, table, lens, want, size)
                lens[:] = [w if all(0 <= p for p in t[:-(-w // size)]) and w <= width * size else x for w, x, t in zip(want, lens, table)]
            elif what == "fork":
                table, lens, copies, _ = pages.fork(refs, table, lens, [g.randint(-1, len(table) - 1) for _ in range(g.randint(1, 6))],
                                                    size, room=g.choice((0, 1)))
            elif what == "free":
                pages.free(refs, table, lens, [g.randint(0, len(table) - 1) for _ in range(2)])
            else:
                flat = [list(t) for t in table]
                pages.compact(refs, flat)
                table = flat
                assert max([p for t in table for p in t], default=-1) < sum(c > 0 for c in refs)
            count = [0] * num
            for t in table:
                for p in t:
                    if p >= 0:
                        count[p] += 1
            assert count == refs
    assert content == {}


def test_beams_by_hand():
    # two beams of three tokens; equal logits are ln 1/3 each
    x = np.zeros((2, 3))
    s, t, p, n, f, _ = beam.select(x, [0.0, -0.5], 2, 4, lengths=[3, 4], eos=2)
    third = np.log(1 / 3)
    assert np.allclose(s, [[third] * 3 + [third - 0.5]]) and t.tolist() == [[0, 1, 2, 0]] and p.tolist() == [[0, 0, 0, 1]]
    assert n.tolist() == [[4, 4, 4, 5]] and f.tolist() == [[0, 0, 1, 0]]
    # a finished beam goes on as itself, then as nothing; a longer one is favoured by alpha 1
    s, t, p, n, f, _ = beam.select(x, [-2.0, -2.0], 2, 2, lengths=[3, 7], finished=[1, 0], eos=2, alpha=1.0)
    assert p.tolist() == [[1, 1]] and np.allclose(s, third - 2)
    s, t, p, n, f, _ = beam.select(x, [-2.0, -np.inf], 2, 3, finished=[1, 0], eos=2)
    assert s.tolist() == [[-2.0, -np.inf, -np.inf]] and t.tolist() == [[2, 0, 1]] and p.tolist() == [[0, 0, 0]]
    assert f.tolist() == [[1, 1, 1]]
    # NaN comes last
    s, t, p, _, _, _ = beam.select([[0.0, np.nan], [-np.inf, -np.inf]], [0.0, 0.0], 2, 3)
    assert p.tolist() == [[1, 1, 0]] and t.tolist() == [[0, 1, 0]] and np.isnan(s[0, 2])
