"""CPU reference of decoding with drafted tokens in float64: a tree's ancestors,
attention under any mask, the verification of chains and trees from given numbers,
and the cache entries that are kept.  Shares no code with the kernels or the
binding."""
from __future__ import annotations

import math

import numpy as np

from oracle import attention as oa

CUT = -1000.0          # log2: tokens less likely by more, beside the likeliest, have weight 0


def ancestors(parents, i):
    """The node itself and its ancestors; a parent that is not an earlier node is none."""
    seen = []
    while i >= 0:
        seen.append(i)
        p = int(parents[i])
        i = p if -1 <= p < i else -1
    return seen


def attend(q, k, v, scale, seen):
    """q [n, H, D], k, v [len, Hk, D] (float64), seen [n, len]: as oracle.attention.attend."""
    n, H, D = q.shape
    Hk = k.shape[1]
    out, av = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, sabs = np.full((n, H), -np.inf), np.zeros((n, H))
    for i in range(n):
        m = np.flatnonzero(seen[i])
        if len(m) == 0:
            continue
        for h in range(H):
            kk, vv = k[m, h // (H // Hk)], v[m, h // (H // Hk)]
            s = kk @ q[i, h] * scale
            top = s.max()
            w = np.exp(s - top)
            lse[i, h] = top + math.log(w.sum())
            w /= w.sum()
            out[i, h], av[i, h] = w @ vv, w @ np.abs(vv)
            sabs[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, av, sabs


def softmax(logits, temperature):
    """Probabilities of one row, None where no token can be."""
    x = np.asarray(logits, dtype=np.float64)
    if x.max() == -np.inf:
        return None
    if not temperature > 0:
        p = np.zeros(len(x))
        p[int(np.argmax(x))] = 1.0
        return p
    t = (x - x.max()) / min(float(temperature), 3.4028234663852886e38)
    w = np.where(t * math.log2(math.e) > CUT, np.exp(t), 0.0)
    return w / w.sum()


def number(u):
    """What a given number counts as."""
    u = np.float32(u)
    if np.isnan(u):
        return 0.0 if np.signbit(u) else 1.0 - 2.0 ** -24
    return min(max(float(u), 0.0), 1.0 - 2.0 ** -24)


def draw(w, u):
    """The lowest index up to which the weights add up to more than u of all, and
    how near (in shares of the whole) u lies to a border."""
    c = np.cumsum(w)
    target = number(u) * c[-1]
    positive = np.flatnonzero(w > 0)
    over = positive[c[positive] > target]
    v = int(over[0]) if len(over) else int(positive[-1])
    borders = np.concatenate([c[positive[positive < v]][-1:], c[v:v + 1] if v != positive[-1] else []])
    return v, float(np.abs(borders - target).min() / c[-1]) if len(borders) else 1.0


def verify_draft(rows, ids, draft, temperature, u, u_draw):
    """One request: rows [n, V] logits, ids [n], draft [n, V] or None.  Returns the
    tokens, the logarithms of their probabilities and the nearest border."""
    tokens, logp, near = [], [], 1.0
    V = rows.shape[1]
    for i in range(len(rows)):
        p = softmax(rows[i], temperature)
        rest = None
        if i + 1 < len(rows):
            x = int(ids[i + 1])
            real = 0 <= x < V and p is not None
            if not temperature > 0:
                stands = real and p[x] > 0
            else:
                q = None if draft is None else softmax(draft[i], temperature)
                if draft is None:
                    qx = 1.0
                    rest = None if p is None else np.where(np.arange(V) == x, 0.0, p)
                elif q is None:
                    real = False
                    qx = 1.0
                else:
                    qx = q[x] if 0 <= x < V else 0.0
                    rest = None if p is None else np.maximum(p - q, 0.0)
                stands = bool(real and number(u[i]) * qx < p[x])
                if real and p[x] > 0:
                    near = min(near, abs(number(u[i]) * qx - p[x]) / p[x])
            if stands:
                tokens.append(x)
                logp.append(math.log(p[x]))
                continue
        if p is None:
            tokens.append(-1)
            logp.append(0.0)
        else:
            w = p if rest is None or not rest.sum() > 0 else rest
            v, gap = draw(w, u_draw)
            if temperature > 0:
                near = min(near, gap)
            tokens.append(v)
            logp.append(math.log(p[v]))
        break
    return tokens, logp, near


def verify_tree(rows, ids, parents, temperature, u):
    """One request: path, tokens, logarithms of their probabilities, nearest border."""
    path, tokens, logp, near = [], [], [], 1.0
    node = 0
    while node is not None:
        p = softmax(rows[node], temperature)
        path.append(node)
        if p is None:
            tokens.append(-1)
            logp.append(0.0)
            break
        v, gap = draw(p, u[node])
        if temperature > 0:
            near = min(near, gap)
        tokens.append(v)
        logp.append(math.log(p[v]))
        node = next((c for c in range(node + 1, len(rows)) if parents[c] == node and ids[c] == v), None)
    return path, tokens, logp, near


def entry(tile, D, token):
    """One token's bytes out of a tile, codes and scales."""
    S = oa.scale_stride(D)
    parts = [tile[(g * oa.PAGE + token) * 16:][:16] for g in range(2 * D // 32)]
    parts += [tile[oa.PAGE * (D + x * S) + token * S:][:S] for x in range(2)]
    return np.concatenate(parts)


def put_entry(tile, D, token, raw):
    S = oa.scale_stride(D)
    for g in range(2 * D // 32):
        tile[(g * oa.PAGE + token) * 16:][:16] = raw[16 * g:16 * g + 16]
    for x in range(2):
        tile[oa.PAGE * (D + x * S) + token * S:][:S] = raw[D + x * S:D + (x + 1) * S]


def keep(cache, D, table, kv_len, n, path, kept):
    """One request's entries in a cache [layers, pages, Hk, tile] (changed in
    place); returns the new length."""
    if not 0 <= kept <= n:
        return kv_len
    before = cache.copy()

    def place(token):
        if token < 0 or token // oa.PAGE >= len(table):
            return None
        page = int(table[token // oa.PAGE])
        return (page, token % oa.PAGE) if 0 <= page < cache.shape[1] else None

    for i in range(kept):
        j = int(path[i])
        if not i < j < n or kv_len - n + i < 0:
            continue
        a, b = place(kv_len - n + j), place(kv_len - n + i)
        if a is None or b is None:
            continue
        for layer in range(cache.shape[0]):
            for h in range(cache.shape[2]):
                put_entry(cache[layer, b[0], h], D, b[1], entry(before[layer, a[0], h], D, a[1]))
    return kv_len - n + kept
