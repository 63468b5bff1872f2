"""One step of a beam search, plain fp64."""

import numpy as np


def select(logits, scores, beams, picks, lengths=None, finished=None, eos=-1, alpha=0.0):
    """logits [rows][vocab] -> (scores, tokens, parents, lengths, finished, gap), [groups][picks]; gap [groups]:
    the smallest difference of neighbouring unequal ranks among the picks and the next one, of different beams
    (where it is large the order is beyond doubt in another precision; equal beams are equal in any)."""
    logits = np.asarray(logits, dtype=np.float64)
    rows, V = logits.shape
    G = rows // beams
    out = [np.zeros((G, picks)) for _ in range(5)]
    gap = np.full(G, np.inf)
    for g in range(G):
        cand = []
        for b in range(beams):
            r = g * beams + b
            x, s0 = logits[r], float(scores[r])
            done = finished is not None and bool(finished[r])
            n = (0 if lengths is None else int(lengths[r])) + (not done)
            if done:
                s = np.full(V, -np.inf)
                s[eos] = s0 if s0 < np.inf else np.nan
                order = [eos] + [v for v in range(min(V, picks + 1)) if v != eos]
            else:
                with np.errstate(invalid="ignore", divide="ignore"):
                    m = x.max()
                    s = s0 + ((x - m) - np.log(np.exp(x - m).sum()))
                if np.isnan(x).any() or (x == np.inf).any() or not s0 < np.inf:
                    s = np.full(V, np.nan)
                elif s0 == -np.inf or m == -np.inf:
                    s = np.full(V, -np.inf)
                order = np.argsort(-x, kind="stable")[:picks] if np.isfinite(s).any() else range(min(V, picks))
            for j, v in enumerate(list(order)[:picks]):
                rank = s[v] / max(n, 1) ** alpha
                cand.append((np.isnan(rank), -rank if not np.isnan(rank) else 0.0, b, j, int(v), s[v], r, n, done))
        cand.sort(key=lambda c: c[:4])
        for k, c in enumerate(cand[:picks]):
            for o, val in zip(out, (c[5], c[4], c[6], c[7], c[8] or c[4] == eos)):
                o[g, k] = val
        for u, v in zip(cand[:picks], cand[1:picks + 1]):
            if u[2] != v[2] and not u[0] and not v[0] and np.isfinite(u[1]) and np.isfinite(v[1]) and v[1] > u[1]:
                gap[g] = min(gap[g], v[1] - u[1])
    return (*out, gap)
