"""Decoding by drafts, in 64 bits and written out plainly: trees of drafted tokens, attention over a cache for them, which drafts the target agrees
to, and the cache with those alone.  Independent of the library: numpy and the cache of `decoder` only."""
import math

import numpy as np

from . import decoder

MOST = 256
MORE = 1 + 2.0 ** -44                 # of q: rounding leaves nothing of p - q where they agree


def follows(parents):
    """Per row the rows that it follows, in order, itself last; nothing for a row that is not there."""
    out = []
    for i, p in enumerate(parents):
        if p == -1:
            out.append([i])
        elif 0 <= p < i and out[p]:
            out.append(out[p] + [i])
        else:
            out.append([])
    return out


def words(rows):
    """[n, 4] uint64: the rows of each set as bits."""
    out = np.zeros((len(rows), MOST // 64), dtype=np.uint64)
    for i, f in enumerate(rows):
        for j in f:
            out[i, j // 64] |= np.uint64(1 << (j % 64))
    return out


def attention(Q, K, V, start, parents, scale, window=0, softcap=0.0):
    """Q [rows, heads, D] of one tree behind `start` tokens; K, V [start + rows, kv_heads, D] -> (o, a) as decoder.attention gives."""
    rows, H, D = Q.shape
    group = H // K.shape[1]
    out, mass = np.zeros((rows, H, D)), np.zeros((rows, H, D))
    for i, f in enumerate(follows(parents)):
        if not f:
            continue
        position = start + len(f) - 1
        keys = [j for j in range(start) if not window or j > position - window] + [start + j for j in f]
        for h in range(H):
            z = K[keys, h // group] @ Q[i, h] * scale
            if softcap:
                z = softcap * np.tanh(z / softcap)
            w = np.exp(z - z.max()) if not np.isnan(z).any() else np.full_like(z, np.nan)
            w = w / w.sum()
            out[i, h], mass[i, h] = w @ V[keys, h // group], w @ np.abs(V[keys, h // group])
    return out, mass


def distribution(x, t):
    """Probabilities of a row of logits at temperature t (t <= 0: all of it at the first of the largest), or None."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or x.max() == np.inf or x.max() == -np.inf:
        return None
    if not t > 0:
        return (np.arange(len(x)) == x.argmax()).astype(np.float64)
    w = np.exp((x - x.max()) / min(max(t, 2.0 ** -100), 2.0 ** 100))
    return w / w.sum()


def held(u):
    """A uniform as it counts."""
    return 0.0 if not u > 0 else min(float(u), 1.0 - 2.0 ** -24)


def verify(logits, draft, tokens, parents, uniforms, t):
    """One sequence.  logits, draft [rows, vocab] (draft: or None) -> (path, next, probs, margin).  margin: how near, relative to the probabilities in question, the nearest
    decision was to going the other way: two computations may differ where it is no more than their error."""
    n, V = logits.shape
    P = [distribution(x, t) for x in logits]
    probs, margin = np.zeros(n), math.inf
    children = [[c for c in range(1, n) if parents[c] == r and r < c] for r in range(n)]
    for r in range(n):
        for c in children[r]:
            if P[r] is not None and 0 <= tokens[c] < V:
                probs[c] = P[r][tokens[c]]
    if n == 0 or parents[0] != -1:                               # a first row that is not there: no row is that could stay
        return [], -1, probs, margin
    r, path = 0, [0]
    while True:
        p, left, stays, without = P[r], 1.0, None, set()
        q = None
        if draft is not None and children[r]:
            q = distribution(draft[r], t) if t > 0 else None
        for c in children[r][:1] if draft is not None else children[r]:
            x, u = tokens[c], held(uniforms[c])
            if p is None or not 0 <= x < V or x in without:
                continue
            if draft is not None and t > 0:
                if q is None:
                    continue
                a, b = u * q[x], p[x]
            else:
                a, b = u * left, p[x]
            if t > 0 and max(a, b) > 0:                          # 0 < 0 is false however it is computed
                margin = min(margin, abs(a - b) / max(a, b))
            if a < b:
                stays = c
                break
            left -= p[x]
            without.add(x)
        if stays is None:
            break
        path.append(stays)
        r = stays
    p = P[r]
    if p is None:
        return path, -1, probs, margin
    if not t > 0:
        return path, int(p.argmax()), probs, margin
    w = p.copy()
    if draft is None:
        w[[x for x in (tokens[c] for c in children[r]) if 0 <= x < V]] = 0.0
    elif children[r] and 0 <= tokens[children[r][0]] < V and q is not None:
        w = np.maximum(p - q * MORE, 0.0)
    if not w.sum() > 0:
        return path, int(np.argmax(logits[r])), probs, margin
    cum = np.cumsum(w)
    goal = held(uniforms[0]) * cum[-1]
    v = int(np.argmax(cum > goal))
    margin = min(margin, 2.0 ** 20 * min(cum[v] - goal, goal - (cum[v] - w[v]) if goal > 0 else math.inf) / cum[-1])      # the sums are in 64 bits: 2^20 times nearer is still far
    return path, v, probs, margin


def keep(cache, pages, start, rows, path):
    """decoder.Cache: the tokens start + path[i] become start + i; a path ends where it does not rise or leaves the rows."""
    good = []
    for r in path:
        if not (good[-1] if good else -1) < r < rows:
            break
        good.append(r)
    P, B = decoder.PAGE, decoder.BLOCK
    codes, scales = cache.codes.copy(), cache.scales.copy()
    at = lambda slot: (pages[slot // P], slot % P, slot % P // B)
    for block in range(start // B, (start + len(good) - 1) // B + 1 if good else 0):
        page, half = pages[block * B // P], block % 2
        moves = {start + i: start + r for i, r in enumerate(good) if (start + i) // B == block}
        earlier = [s for s in range(block * B, block * B + B) if s < start]
        for h in range(codes.shape[1]):
            for which in (0, 1):
                exps = [int(scales[at(s)[0], h, which, at(s)[2]]) - 127 for s in list(moves.values()) + earlier]
                e = max(exps)
                for s in earlier:
                    moves[s] = s
                for dst, src in moves.items():
                    p, i, b = at(src)
                    was = int(scales[p, h, which, b]) - 127
                    code = codes[p, h, which, i]
                    rounded = np.where(code & 0x7F == 0x7F, code, decoder.e4m3_encode(decoder.e4m3_decode(code) * 2.0 ** (was - e)))      # a NaN's code stays, of either sign
                    cache.codes[page, h, which, dst % P] = code if was == e else rounded
                for s in earlier:
                    del moves[s]
                cache.scales[page, h, which, half] = e + 127
    return len(good)
