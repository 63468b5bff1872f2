"""Between the linears of a decoder layer, plain fp64: attention over given
keys, rotary positions, routing, residual and norms.  Loops over tokens and
heads; nothing is paged, tiled or fused."""

import numpy as np


# ------------------------------------------------------------------ attention

def visible(n, p, causal=True, window=0):
    """Keys that a token at position p of n keys sees, as a boolean [n]."""
    j = np.arange(n)
    see = np.ones(n, dtype=bool)
    if causal:
        see &= j <= p
    if window:
        see &= j > p - window
    return see


def attend(q, k, v, scale, causal=True, window=0):
    """One sequence: q [a][Hq][D] at the last a positions of n keys k, v
    [Hkv][n][D].  Returns (o [a][Hq][D], lse [a][Hq], weight [a][Hq][D], most
    [a][Hq]): weight is sum p |v| / sum p and most the largest
    scale sum |q k| of a seen key (what rounding errors scale with)."""
    a, Hq, D = q.shape
    n = k.shape[1]
    o, weight = np.zeros((a, Hq, D)), np.zeros((a, Hq, D))
    lse, most = np.full((a, Hq), -np.inf), np.zeros((a, Hq))
    for i in range(a):
        see = visible(n, n - a + i, causal, window)
        if not see.any():
            continue
        for h in range(Hq):
            kk, vv = k[h * k.shape[0] // Hq][see], v[h * k.shape[0] // Hq][see]
            s = scale * (kk @ q[i, h])
            m = s.max()
            e = np.exp(s - m)
            o[i, h] = e @ vv / e.sum()
            weight[i, h] = e @ np.abs(vv) / e.sum()
            lse[i, h] = m + np.log(e.sum())
            most[i, h] = (abs(scale) * (np.abs(kk) @ np.abs(q[i, h]))).max()
    return o, lse, weight, most


# ------------------------------------------------------------ rotary positions

def rotate(x, pos, inv_freq, interleaved=False, magnitude=1.0):
    """x [heads][D] at position pos, its first 2 len(inv_freq) values turned."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    for j in range(half):
        lo, hi = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = magnitude * np.cos(pos * float(inv_freq[j])), magnitude * np.sin(pos * float(inv_freq[j]))
        u, w = x[:, lo].copy(), x[:, hi].copy()
        x[:, lo], x[:, hi] = u * c - w * s, u * s + w * c
    return x


def head_norm(x, weight, eps):
    """x [heads][D] by each head's root mean square."""
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps) * weight


# -------------------------------------------------------------------- routing

def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0):
    """logits [T][E] -> (ids [T][k], weights [T][k], gap [T]): gap is the
    smallest difference between neighbours among the values that decided (ids
    are beyond doubt in another precision where it is large)."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    ids, w, gap = np.zeros((T, k), dtype=np.int64), np.zeros((T, k)), np.full(T, np.inf)
    for t in range(T):
        x = logits[t]
        if score == "softmax":
            m = np.max(x)
            p = np.zeros(E) if m == -np.inf else np.exp(x - m) / np.sum(np.exp(x - m))
        else:
            p = 1.0 / (1.0 + np.exp(-x))
        c = x if bias is None else p + bias
        open_ = list(range(E))
        if groups > 1:
            size = E // groups
            src = p if bias is None and group_best == 2 else c
            best = [sum(sorted(src[g * size:(g + 1) * size])[::-1][:group_best]) for g in range(groups)]
            order = sorted(range(groups), key=lambda g: (-best[g], g))
            if top_groups < groups:
                gap[t] = min(gap[t], best[order[top_groups - 1]] - best[order[top_groups]])
            open_ = [e for e in range(E) if e // size in order[:top_groups]]
        order = sorted(open_, key=lambda e: (-c[e], e))
        ids[t] = order[:k]
        for u, v in zip(order[:k], order[1:k + 1]):
            gap[t] = min(gap[t], c[u] - c[v])
        w[t] = p[ids[t]]
        if renormalize and w[t].sum() != 0:
            w[t] /= w[t].sum()
        w[t] *= scale
    return ids, w, gap


# ---------------------------------------------------------- residual and norms

def normalise(x, kind, eps):
    x = np.asarray(x, dtype=np.float64)
    if kind == "layer":
        x = x - np.mean(x, axis=-1, keepdims=True)
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def residual_norm(y, weight, residual=None, slot_weights=None, post_weight=None, gate=None, bias=None, kind="rms",
                  eps=1e-6, alpha=1.0, beta=1.0):
    """(h, out), both [T][d]."""
    u = np.asarray(y, dtype=np.float64)
    if slot_weights is not None:
        u = np.sum(u * np.asarray(slot_weights, dtype=np.float64)[:, :, None], axis=1)
    if post_weight is not None:
        u = normalise(u, kind, eps) * post_weight
    if gate is not None:
        u = u * gate
    h = beta * u
    if residual is not None:
        h = h + alpha * np.asarray(residual, dtype=np.float64)
    out = normalise(h, kind, eps) * weight
    return h, out if bias is None else out + bias
