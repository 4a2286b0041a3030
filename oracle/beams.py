"""A beam search over resident histories in 64 bits: the selection of beams, the reordering of a
cache's sequences, and attention to a prefix that continuations share.  Plain numpy and Python lists, from the
definitions alone.
"""
import math

import numpy as np

from .history import attend


def log_sum(z):
    """(m, log of the sum of exp(z - m)) over the finite numbers of z, m the largest of them (None: there are none).  Apart,
    since next to a large m their sum would lose the logarithm."""
    z = np.array([float(x) for x in z if math.isfinite(x)])
    if not len(z):
        return None, 0.0
    return z.max(), math.log(math.fsum(np.exp(z - z.max())))


def select(logits, beams, keep, score=None, done=None, allowed=None, eos=-1, in_place=False):
    """logits [requests * beams, V], score and done [requests, beams], allowed truth values
    [requests * beams, V].  Returns (parent, token, value in 64 bits, done), each [requests, keep]."""
    logits = np.asarray(logits, dtype=np.float64)
    R = logits.shape[0] // beams
    parent = np.full((R, keep), -1, dtype=np.int64)
    token = np.full((R, keep), -1, dtype=np.int64)
    value = np.full((R, keep), -np.inf)
    ends = np.zeros((R, keep), dtype=np.uint8)
    for r in range(R):
        found = []   # (-value, beam, token)
        for b in range(beams):
            n = r * beams + b
            s = 0.0 if score is None else float(score[r][b])
            if not math.isfinite(s):
                continue
            if done is not None and done[r][b]:
                found.append((-s, b, max(eos, 0)))
                continue
            m, total = log_sum(logits[n])
            if m is None:
                continue
            base = s - total
            ok = np.isfinite(logits[n])
            if allowed is not None:
                ok = ok & allowed[n]
            v = np.flatnonzero(ok)
            c = base + (logits[n][v] - m)
            best = np.lexsort((v, -c))[:keep]
            found += [(-float(c[i]), b, int(v[i])) for i in best]
        found = sorted(found)[:keep]
        places = list(range(keep))
        if in_place:
            kept = {b for _, b, _ in found}
            free = [p for p in range(keep) if p not in kept]
            places, headed = [], set()
            for _, b, _ in found:
                places.append(free.pop(0) if b in headed else b)
                headed.add(b)
        for p, (c, b, v) in zip(places, found):
            was = bool(done is not None and done[r][b])
            parent[r, p], value[r, p] = b, -c
            token[r, p] = eos if was else v
            ends[r, p] = was or v == eos
    return parent, token, value, ends


def reorder(cache, offset, parent, max_members=1024):
    """cache: history.Cache; parent counted from sequence offset[0]."""
    old = [(list(t), n, list(k), list(v)) for t, n, k, v in zip(cache.table, cache.len, cache.k, cache.v)]
    for first, end in zip(offset, offset[1:]):
        n = min(end - first, max_members)
        for i in range(n):
            s, m = first + i, first + i - offset[0]
            p = parent[m] if m < len(parent) else i
            if p == i or p >= n:
                continue
            for page in old[s][0]:
                if page is not None:
                    cache.refs[page] -= 1
            table, length, k, v = old[first + p] if p >= 0 else ([], 0, [], [])
            cache.table[s], cache.len[s] = list(table), length
            cache.k[s], cache.v[s], cache.fresh[s] = list(k), list(v), 0
            for page in table:
                if page is not None:
                    cache.refs[page] += 1


def attend_prefix(cache, prefix, s, layer, q, causal, window=0, sinks=0, scale=None):
    """Queries q [n, H, D] of member s over sequence `prefix` (-1: none) and its own tokens."""
    parts = [cache.values(x, layer) + (cache.len[x],) for x in (prefix, s) if x >= 0 and cache.len[x] > 0]
    n, own = q.shape[0], cache.len[s]
    L = cache.len[prefix] if prefix >= 0 else 0
    if not parts:
        none = np.zeros((0, 1, q.shape[2]))
        return attend(q, none, none, np.zeros((n, 0), dtype=bool), scale)
    k, v, held = (np.concatenate([p[i] for p in parts]) for i in range(3))
    place = (own - n + np.arange(n) if causal else np.full(n, own))[:, None]
    j = np.arange(L + own)[None, :]
    see = held[None] & ((j < L) | (j - L <= place))
    if window > 0:
        see &= (L + place - j < window) | (j < sinks)
    return attend(q, k, v, see, scale)
