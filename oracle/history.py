"""Attention over whole histories in 64 bits: causal attention with a window and sink tokens, and the
paged 8-bit cache of keys and values (what each block stands for, which pages each call
takes and gives back).  Plain numpy and Python lists, from the definitions alone.
"""
import numpy as np

PAGE = 64
TINY = 2.0 ** -100


def visible(pos, length, window=0, sinks=0):
    """[len(pos), length] truth values: the tokens that a query at each position sees."""
    pos = np.asarray(pos, dtype=np.int64)[:, None]
    j = np.arange(length, dtype=np.int64)[None, :]
    see = j <= pos
    if window > 0:
        see &= (pos - j < window) | (j < sinks)
    return see


def attend(q, k, v, see, scale=None):
    """q [n, H, D], k and v [L, Hkv, D], see [n, L] -> out [n, H, D], lse [n, H] and, for error
    bounds, size [n, H, D] = sum of weights times |v| and reach [n, H] = the largest
    scale * sum |q k| of a seen token.  Nothing seen: zeros and -inf."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, H, D = q.shape
    G = H // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out, size = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, reach = np.full((n, H), -np.inf), np.zeros((n, H))
    if k.shape[0] == 0:
        return out, lse, size, reach
    some = see.any(1)
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        s = np.where(see, scale * (q[:, h] @ kh.T), -np.inf)
        m = np.where(some, s.max(1), 0.0)
        p = np.exp(s - m[:, None])
        z = p.sum(1)
        p /= np.where(some, z, 1.0)[:, None]
        out[:, h], size[:, h] = p @ vh, p @ np.abs(vh)
        with np.errstate(divide="ignore"):
            lse[:, h] = m + np.log(z)
        reach[:, h] = np.where(see, scale * (np.abs(q[:, h]) @ np.abs(kh).T), 0.0).max(1)
    return out, lse, size, reach


def window_attention(q, k, v, window=0, sinks=0, scale=None):
    """One sequence attends to itself."""
    L = q.shape[0]
    return attend(q, k, v, visible(np.arange(L), L, window, sinks), scale)


def quantise(x):
    """(codes, scale) of one block and head [64, D]: 127 x / max|x| rounded half to even, and
    max|x| / 127; zeros and 1 below TINY."""
    x = np.asarray(x, dtype=np.float64)
    top = np.abs(x).max()
    if not top >= TINY:
        return np.zeros(x.shape, dtype=np.int64), 1.0
    # for values of at most 24 bits 127 x is exact, and a quotient that is no half is not rounded to one
    return np.rint(127.0 * x / top).astype(np.int64), top / 127.0


class Cache:
    """The cache's state as plain values: tokens[s] a list of (k [layers, H, D], v), of which
    those of full blocks are taken through quantise(); table[s] the pages (None: released)."""

    def __init__(self, seqs, pages, max_blocks, layers=1):
        self.table = [[] for _ in range(seqs)]
        self.k = [[] for _ in range(seqs)]     # per sequence: [layers, H, D] per token
        self.v = [[] for _ in range(seqs)]
        self.refs = [0] * pages
        self.fresh = [0] * seqs
        self.max_blocks, self.layers = max_blocks, layers
        self.len = [0] * seqs

    def extend(self, count):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        dry = False
        self.fresh = [0] * len(count)
        for s, n in enumerate(count):
            if n <= 0 or (self.len[s] + n) // PAGE > self.max_blocks:
                continue
            need = (self.len[s] + n) // PAGE - self.len[s] // PAGE
            dry = dry or need > len(free)
            if dry:
                continue
            for p in free[:need]:
                self.refs[p] = 1
            self.table[s] += free[:need]
            free = free[need:]
            self.fresh[s] = n
            self.len[s] += n

    def append(self, k, v, offset):
        """k, v [layers, rows, H, D]."""
        for s, n in enumerate(self.fresh):
            for i in range(offset[s], offset[s] + n):
                self.k[s].append(np.array(k[:, i], dtype=np.float64))
                self.v[s].append(np.array(v[:, i], dtype=np.float64))

    def values(self, s, layer):
        """Keys and values [len, H, D] that sequence s stands for, and which tokens are held."""
        out = []
        for rows in (self.k[s], self.v[s]):
            if not rows:
                out.append(np.zeros((0, 1, 1)))
                continue
            x = np.stack([r[layer] for r in rows])
            for a in range(0, len(rows) // PAGE * PAGE, PAGE):
                for h in range(x.shape[1]):
                    codes, scale = quantise(x[a:a + PAGE, h])
                    x[a:a + PAGE, h] = codes * scale
            out.append(x)
        held = np.ones(self.len[s], dtype=bool)
        for b, p in enumerate(self.table[s]):
            if p is None:
                held[b * PAGE:(b + 1) * PAGE] = False
        return out[0], out[1], held

    def fork(self, parent):
        was = list(self.len)
        for s, p in enumerate(parent):
            if not 0 <= p < len(parent) or parent[p] >= 0 or was[s] != 0:
                continue
            self.table[s], self.len[s], self.fresh[s] = list(self.table[p]), self.len[p], 0
            self.k[s], self.v[s] = list(self.k[p]), list(self.v[p])
            for page in self.table[s]:
                if page is not None:
                    self.refs[page] += 1

    def _release(self, s, b):
        if self.table[s][b] is not None:
            self.refs[self.table[s][b]] -= 1
            self.table[s][b] = None

    def free(self, drop):
        for s, d in enumerate(drop):
            if d:
                for b in range(len(self.table[s])):
                    self._release(s, b)
                self.table[s], self.k[s], self.v[s] = [], [], []
                self.len[s] = self.fresh[s] = 0

    def trim(self, window, sinks):
        for s in range(len(self.len)):
            for b in range(len(self.table[s])):
                if b * PAGE >= sinks and (b + 1) * PAGE <= self.len[s] - window + 1:
                    self._release(s, b)

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] == 0]
        to = dict(zip([p for p in used if p >= U], holes))
        for p, q in to.items():
            self.refs[q], self.refs[p] = self.refs[p], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return U

    def attend(self, s, layer, q, causal, window=0, sinks=0, scale=None):
        k, v, held = self.values(s, layer)
        n, L = q.shape[0], self.len[s]
        pos = L - n + np.arange(n) if causal else np.full(n, L)
        if L == 0:
            k = v = np.zeros((0, 1, q.shape[2]))
        return attend(q, k, v, visible(pos, L, window, sinks) & held[None], scale)
