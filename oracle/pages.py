"""Pages and their holders, plain loops over lists: a pool's counts, tables whose
entries outside of it hold nothing, and the copies that a call makes.  Every
function returns the copies [(from, to)] and how many entries got no page."""


def _own(kv_len, prefix, width, size):
    return min(max(kv_len - prefix, 0), width * size)


def _held(p, refs):
    return 0 <= p < len(refs)


def fork(refs, table, kv_len, parents, size, room=0, prefix=0):
    """(new table, new kv_len, copies, missing); refs changes in place."""
    width, n = len(table[0]), len(table)
    children = [[i for i, p in enumerate(parents) if p == r] for r in range(n)]
    for r in range(n):
        used = -(-_own(kv_len[r], prefix, width, size) // size)
        for e, p in enumerate(table[r]):
            if _held(p, refs):
                refs[p] += len(children[r]) - 1 if e < used else 0 if children[r] else -1
    new, lens = [], []
    for i, r in enumerate(parents):
        if not 0 <= r < n:
            new.append([-1] * width), lens.append(0)
            continue
        used = -(-_own(kv_len[r], prefix, width, size) // size)
        first = children[r][0] == i
        new.append([p if _held(p, refs) and (e < used or first) else -1 for e, p in enumerate(table[r])])
        lens.append(max(kv_len[r], 0))
    want = [x + room if 0 <= r < n else 0 for x, r in zip(lens, parents)]
    copies, missing = _give(refs, new, lens, want, size, prefix) if room else ([], 0)
    return new, lens, copies, missing


def reserve(refs, table, kv_len, want, size, prefix=0):
    return _give(refs, table, kv_len, want, size, prefix)


def _give(refs, table, kv_len, want, size, prefix):
    """A growing row copies a partly used last page that others hold too, but where all its holders grow the first
    keeps it; then it gets what it lacks.  Where pages run out the row keeps the one it holds."""
    width = len(table[0])
    asks, missing = [], 0
    growing = {}
    for i, row in enumerate(table):
        own = _own(kv_len[i], prefix, width, size)
        if want[i] > kv_len[i] and own % size:
            growing.setdefault(row[-(-own // size) - 1], []).append(i)
    for i, row in enumerate(table):
        own = _own(kv_len[i], prefix, width, size)
        used = -(-own // size)
        if want[i] <= kv_len[i]:
            continue
        need = max(-(-max(want[i] - prefix, 0) // size), used)
        missing += min(max(need - width, 0), 1024)
        if own % size and _held(row[used - 1], refs):
            who = growing[row[used - 1]]
            if len(who) != refs[row[used - 1]] or who[0] != i:
                asks.append((i, used - 1, row[used - 1]))
        asks += [(i, e, None) for e in range(used, min(need, width)) if not _held(row[e], refs)]
    free = [p for p, c in enumerate(refs) if c == 0]
    copies = []
    for k, (i, e, old) in enumerate(asks):
        page = free[k] if k < len(free) else -1
        missing += page < 0
        if page >= 0:
            refs[page] = 1
            if old is not None:
                refs[old] -= 1
                copies.append((old, page))
        if page >= 0 or old is None:
            table[i][e] = page
    return copies, missing


def free(refs, table, kv_len, rows):
    for r in rows:
        if 0 <= r < len(table):
            for e, p in enumerate(table[r]):
                if _held(p, refs):
                    refs[p] -= 1
                table[r][e] = -1
            kv_len[r] = 0


def compact(refs, tables):
    """tables: flat lists."""
    live = sum(c > 0 for c in refs)
    movers = [p for p in range(live, len(refs)) if refs[p] > 0]
    holes = [p for p in range(live) if refs[p] <= 0]
    name = dict(zip(movers, holes))
    for f, t in name.items():
        refs[t], refs[f] = refs[f], 0
    for t in tables:
        for e, p in enumerate(t):
            if live <= p < len(refs):
                t[e] = name.get(p, -1)
    return list(name.items())
