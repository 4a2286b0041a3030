"""The performance cases of attention over whole histories: the windowed attention of packed
histories (`attend_window`) and the paged 8-bit cache of their keys and values (`KvCache`,
`kv_extend`, `kv_append`, `kv_attend`, `kv_fork`, `kv_free`, `kv_trim`, `kv_compact`).

A case's `kind`:
  window   attend_window: a batch of histories attends to itself
  attend   kv_attend: candidates, single new tokens or chunks of them over resident histories
  ingest   kv_extend + kv_append + kv_attend + kv_free: whole histories enter the cache, are
           scored against once and leave
  slate    kv_fork + kv_extend + kv_append + kv_attend + kv_free: continuations of resident
           histories
  fork     kv_fork + kv_trim on restored page tables
  compact  kv_compact on restored page tables

Where `own` is false, run() computes the same in elementary torch operations in 32 bits on the
same buffers.  Lengths are those of this repository's workloads (1024 to 16384 actions, hundreds of
candidates, heads of 32 or 64 features), spread evenly over a case's range.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

P = 64                 # tokens of a page
TINY = 2.0 ** -100     # a block below this is stored as zeros
NONE, CAUSAL = 1, 0    # masks, as the library's flags


# ------------------------------------------------------------------------- cases
def _window(name, dtype, R, L_min, L, heads, kv_heads, D, window, sinks):
    c = dict(kind="window", dtype=dtype, R=R, L_min=L_min, L=L, heads=heads, kv_heads=kv_heads,
             D=D, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _attend(name, S, L_min, L, n_min, n, heads, kv_heads, D, mask, window=0, sinks=0):
    c = dict(kind="attend", S=S, L_min=L_min, L=L, n_min=n_min, n=n, heads=heads,
             kv_heads=kv_heads, D=D, mask=mask, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _ingest(name, S, L_min, L, n, heads, kv_heads, D):
    c = dict(kind="ingest", S=S, L_min=L_min, L=L, n=n, heads=heads, kv_heads=kv_heads, D=D)
    return dict(c, name=name) if name else c


def _slate(name, S, C, L_min, L, m, heads, kv_heads, D, window=0, sinks=0):
    c = dict(kind="slate", S=S, C=C, L_min=L_min, L=L, m=m, heads=heads, kv_heads=kv_heads, D=D,
             window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _fork(name, S, C, L_min, L, layers, kv_heads, D, window, sinks):
    c = dict(kind="fork", S=S, C=C, L_min=L_min, L=L, layers=layers, kv_heads=kv_heads, D=D,
             window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _compact(name, S, L_min, L, layers, kv_heads, D, free):
    """`free`: share of the pool's pages that are free, scattered among the used ones."""
    c = dict(kind="compact", S=S, L_min=L_min, L=L, layers=layers, kv_heads=kv_heads, D=D,
             free=free)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one long history encodes itself: the last 1024 actions and the first 4
        _window("history_16k", "bf16", 1, 16384, 16384, 4, 4, 64, 1024, 4),
        # a batch of users with histories of very different lengths, whole causal attention
        _window("history_batch", "bf16", 32, 203, 4000, 4, 2, 64, 0, 0),
        # the same in fp32 (parity runs, small deployments), odd lengths, a short window
        _window("history_f32", "f32", 8, 57, 1000, 8, 8, 32, 200, 1),
        # one candidate against one long history: the smallest call, latency
        _attend("score_one", 1, 16384, 16384, 1, 1, 4, 4, 64, NONE),
        # one ranking request: 1000 candidates against the whole 16384-action history
        _attend("score_request", 1, 16384, 16384, 1000, 1000, 4, 4, 64, NONE),
        # one new action for each of 64 users, shared key heads
        _attend("new_action", 64, 1024, 16384, 1, 1, 8, 2, 64, CAUSAL),
        # a few candidates for each of 48 users within a window, wide heads
        _attend("score_window", 48, 700, 16384, 1, 24, 8, 4, 128, NONE, 2000, 7),
        # whole histories enter the cache and serve one candidate each
        _ingest("ingest", 64, 1024, 16384, 1, 4, 4, 64),
        # one short history enters it: latency
        _ingest("ingest_one", 1, 333, 333, 5, 4, 4, 64),
        # slates of 5 items that continue 16 resident histories, 8 slates each
        _slate("slate", 16, 8, 1024, 16384, 5, 4, 4, 64),
        # 512 forks of 32 histories, then every sequence keeps a window
        _fork("fork_trim", 32, 16, 1000, 16384, 2, 4, 64, 4096, 4),
        # half of a pool is free in scattered pages and is handed back
        _compact("compact", 32, 1024, 16384, 2, 4, 64, 0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window", "window", "attend", "attend", "attend", "ingest", "slate", "fork",
                       "compact"])
    D = rng.choice([32, 64, 64, 128])
    kv_heads = rng.choice([1, 2, 4])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    low = rng.choice([1.0, 0.5, 0.06])
    if kind == "window":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        L = _log(rng, 20, 16384 if dtype == "bf16" else 2000)
        most = 8e8 * min(1.0, 64 / D)   # scores that the plain form holds
        if L * L * heads > most:
            heads, kv_heads, D = 2, rng.choice([1, 2]), 64
        R = _log(rng, 1, max(1, min(64, int(most / (L * L * heads)))))
        window = rng.choice([0, _log(rng, 1, 4000)])
        return _window(None, dtype, R, max(1, int(L * low)), L, heads, kv_heads, D, window,
                       rng.choice([0, 1, 4, 70]) if window else 0)
    if kind == "attend":
        L = _log(rng, 20, 16384)
        S = _log(rng, 1, max(1, min(64, int(2e8 / (L * kv_heads * D)))))
        n = _log(rng, 1, max(1, min(1000, int(6e7 / (S * L * heads) * min(1.0, 64 / D)))))
        window = rng.choice([0, 0, _log(rng, 1, 4000)])
        return _attend(None, S, max(1, int(L * low)), L, rng.choice([1, n]), n, heads, kv_heads, D,
                       rng.choice([NONE, CAUSAL]), window, rng.choice([0, 4, 70]) if window else 0)
    L = _log(rng, 100, 16384)
    if kind == "ingest":
        return _ingest(None, _log(rng, 1, max(1, min(64, 1000000 // L))), max(1, int(L * low)), L,
                       rng.randint(1, 8), kv_heads, kv_heads, min(D, 64))
    S = _log(rng, 1, max(1, min(32, 400000 // L)))
    if kind == "slate":
        return _slate(None, S, rng.randint(1, 8), max(1, int(L * low)), L, _log(rng, 1, 100),
                      kv_heads, kv_heads, min(D, 64))
    if kind == "fork":
        return _fork(None, S, rng.randint(1, 16), max(1, int(L * low)), L, rng.choice([1, 2]),
                     kv_heads, min(D, 64), _log(rng, 100, 8000), rng.choice([0, 4, 70]))
    return _compact(None, S, max(1, int(L * low)), L, rng.choice([1, 2]), kv_heads, min(D, 64),
                    rng.uniform(0.1, 0.8))


def spread(lo, hi, n):
    """n whole numbers spread evenly over lo..hi, in an order of no pattern."""
    v = [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(n * 1000003 + hi).shuffle(v)
    return v


# ------------------------------------------------------------------------- work
def _visible(n_keys, pos, window, sinks):
    """Keys that a query at `pos` sees of n_keys."""
    top = min(n_keys, pos + 1)
    if window == 0 or top <= 0:
        return max(0, top)
    lo = max(0, pos - window + 1)
    return max(0, top - lo) + min(sinks, lo, top)


def _attend_work(lens, counts, heads, kv_heads, D, mask, window, sinks):
    """Bytes and operations of kv_attend: every key that some query sees, once."""
    keys = pairs = 0
    for L, n in zip(lens, counts):
        if n == 0:
            continue
        first = L - n if mask == CAUSAL else L
        last = L - 1 if mask == CAUSAL else L
        lo = max(0, first - window + 1) if window else 0
        keys += L - lo + min(sinks, lo)
        if mask == NONE:
            pairs += n * _visible(L, last, window, sinks)
        else:
            pairs += sum(_visible(L, first + i, window, sinks) for i in range(n))
    rows = sum(counts)
    return {"bytes": keys * kv_heads * (2 * D + 8 / P) + rows * heads * (4 * D + 4),
            "flops": 4.0 * D * heads * pairs}


def work(case):
    c = SimpleNamespace(**case)
    if c.kind == "window":
        lens = spread(c.L_min, c.L, c.R)
        w = c.window
        pairs = 0
        for L in lens:   # rows below the window see all before them, the others w and the sinks
            full = L if w == 0 else min(L, w)
            pairs += full * (full + 1) // 2
            if L > full:
                pairs += (L - full) * w + sum(min(c.sinks, i + 1) for i in range(min(L - full, c.sinks + 1)))
                pairs += max(0, L - full - c.sinks - 1) * c.sinks
        es = 2 if c.dtype == "bf16" else 4
        rows = sum(lens)
        return {"bytes": rows * c.D * es * 2 * (c.heads + c.kv_heads) + rows * c.heads * 4,
                "flops": 4.0 * c.D * c.heads * pairs}
    lens = spread(c.L_min, c.L, c.S)
    if c.kind == "attend":
        return _attend_work(lens, spread(c.n_min, c.n, c.S), c.heads, c.kv_heads, c.D, c.mask,
                            c.window, c.sinks)
    token = 2 * c.kv_heads * c.D   # values of a token's keys and values
    if c.kind == "ingest":
        a = _attend_work(lens, [c.n] * c.S, c.heads, c.kv_heads, c.D, NONE, 0, 0)
        return {"bytes": a["bytes"] + sum(lens) * token * 3, "flops": a["flops"]}
    if c.kind == "slate":
        # a parent's pages are read once for all of its slates; the tails are copied
        a = _attend_work(lens, [c.C * c.m] * c.S, c.heads, c.kv_heads, c.D, NONE, c.window, c.sinks)
        tails = sum(L % P for L in lens) * c.C * token * 4
        return {"bytes": a["bytes"] + tails + c.S * c.C * c.m * token * 4, "flops": a["flops"]}
    if c.kind == "fork":
        tails = sum(L % P for L in lens) * c.C * token * 4 * c.layers
        blocks = sum(L // P for L in lens)
        return {"bytes": tails + blocks * 4 * (1 + c.C) + blocks * (1 + c.C) * 8, "flops": 0}
    pages, used = _pool(c, lens)
    moved = used - int(used * used / pages)   # used pages that lie behind the used count
    return {"bytes": moved * c.layers * c.kv_heads * (2 * P * c.D + 8) * 2 + pages * 8, "flops": 0}


def _pool(c, lens):
    used = sum(L // P for L in lens)
    return max(used + 1, int(used / (1 - c.free))), used


# ------------------------------------------------------------------------- inputs
def _quantise(x):
    """(codes int8, scale) of x [..., P, D]: one scale for the last two axes.  For values of 8
    significant bits 127 x is exact and its quotient rounds to a half only where it is one."""
    top = x.abs().amax((-2, -1), keepdim=True)
    small = top < TINY
    top = torch.where(small, torch.full_like(top, 127.0), top)
    n = torch.full_like(top, 127.0)
    codes = torch.round(x * n / top).clamp(-127, 127)
    codes = torch.where(small, torch.zeros_like(codes), codes)
    return codes.to(torch.int8), (top / n)[..., 0, 0]


def _cache(g, layers, pages, seqs, kv_heads, D, max_blocks, meta, fill=True):
    """A cache's buffers; pages and tails hold random tokens (values wider in some features than
    in others, as projections give), or nothing yet."""
    dev = "cuda"
    shape = (layers, pages, kv_heads, P, D)
    t = SimpleNamespace(
        k=torch.zeros(shape, dtype=torch.int8, device=dev),
        v=torch.zeros(layers, pages, kv_heads, D, P, dtype=torch.int8, device=dev),
        k_scale=torch.ones(layers, pages, kv_heads, device=dev),
        v_scale=torch.ones(layers, pages, kv_heads, device=dev),
        k_tail=torch.zeros(layers, seqs, kv_heads, P, D, dtype=torch.bfloat16, device=dev),
        v_tail=torch.zeros(layers, seqs, kv_heads, D, P, dtype=torch.bfloat16, device=dev))
    if fill:
        wide = torch.exp(0.5 * torch.randn(kv_heads, 1, D, generator=g, device=dev))
        for layer in range(layers):
            t.k[layer], t.k_scale[layer] = _quantise(
                torch.randn(shape[1:], generator=g, device=dev) * wide)
            v, t.v_scale[layer] = _quantise(torch.randn(shape[1:], generator=g, device=dev) * wide)
            t.v[layer] = v.transpose(-1, -2)
            t.k_tail[layer] = torch.randn(t.k_tail.shape[1:], generator=g, device=dev) * wide
            t.v_tail[layer] = torch.randn(t.v_tail.shape[1:], generator=g, device=dev)
    # page tables, lengths, tokens of the last extension and holders of each page, in one buffer
    n = seqs * max_blocks
    t.meta = meta.to(device=dev, dtype=torch.int32)
    t.table = t.meta[:n].view(seqs, max_blocks)
    t.length = t.meta[n:n + seqs]
    t.fresh = t.meta[n + seqs:n + 2 * seqs]
    t.refs = t.meta[n + 2 * seqs:]
    return t


def _tables(lens, seqs, max_blocks, pages, seed):
    """[table | length | fresh | refs]: the first sequences hold `lens` tokens on pages that lie
    anywhere in the pool."""
    r = torch.Generator().manual_seed(seed)
    ids = torch.randperm(pages, generator=r)
    table = torch.full((seqs, max_blocks), -1, dtype=torch.int64)
    refs = torch.zeros(pages, dtype=torch.int64)
    at = 0
    for s, L in enumerate(lens):
        n = L // P
        table[s, :n] = ids[at:at + n]
        at += n
    refs[ids[:at]] = 1
    length = torch.tensor(list(lens) + [0] * (seqs - len(lens)))
    return torch.cat([table.view(-1), length, torch.zeros(seqs, dtype=torch.int64), refs])


def _offsets(counts):
    o = [0]
    for n in counts:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int64, device="cuda"), o[-1]


def _rows(g, n, heads, D, dtype=torch.bfloat16):
    return torch.randn(n, heads, D, generator=g, device="cuda").to(dtype)


def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = SimpleNamespace(case=c)
    if c.kind == "window":
        lens = spread(c.L_min, c.L, c.R)
        offset, total = _offsets(lens)
        dt = torch.bfloat16 if c.dtype == "bf16" else torch.float32
        # one projection's output: a row holds its queries, keys and values
        qkv = _rows(g, total, c.heads + 2 * c.kv_heads, c.D, dt)
        st.q, st.k, st.v = qkv.split([c.heads, c.kv_heads, c.kv_heads], 1)
        st.offset = offset[:-1].contiguous()
        st.length = torch.tensor(lens, dtype=torch.int32, device="cuda")
        st.out = torch.empty(total, c.heads, c.D, dtype=dt, device="cuda")
        st.lse = torch.empty(total, c.heads, device="cuda")
        return st
    lens = spread(c.L_min, c.L, c.S)
    pages = sum(L // P for L in lens)
    layers = getattr(c, "layers", 1)
    blocks = c.L // P + 3
    seqs, counts, new = c.S, None, None
    if c.kind == "attend":
        counts = spread(c.n_min, c.n, c.S)
        pages += 7
    elif c.kind == "ingest":
        counts, new = [c.n] * c.S, lens
        pages += 7
    elif c.kind == "slate":
        seqs = c.S * (1 + c.C)
        counts = new = [0] * c.S + [c.m] * (c.S * c.C)
        pages += c.S * c.C * (c.m // P + 1)
    elif c.kind == "fork":
        seqs = c.S * (1 + c.C)
        pages += 7
    else:
        pages = _pool(c, lens)[0]
    blocks += max(new or [0]) // P
    meta = _tables([] if c.kind == "ingest" else lens, seqs, blocks, pages, seed)
    st.c = _cache(g, layers, pages, seqs, c.kv_heads, c.D, blocks, meta, c.kind != "ingest")
    st.c.max_len = c.L + (max(new) if c.kind == "slate" else 0)
    if new is not None:
        st.count = torch.tensor(new, dtype=torch.int32, device="cuda")
        st.new_offset, total = _offsets(new)
        st.new_max = max(new)
        st.k, st.v = _rows(g, total, 2 * c.kv_heads, c.D).split([c.kv_heads, c.kv_heads], 1)
        st.drop = (torch.tensor(new, device="cuda") > 0).to(torch.uint8)
    if counts is not None:
        st.offset, total = _offsets(counts)
        st.n = max(counts)
        st.q = _rows(g, total, c.heads, c.D) * 1.5
        st.out = torch.empty(total, c.heads, c.D, dtype=torch.bfloat16, device="cuda")
        st.lse = torch.empty(total, c.heads, device="cuda")
    if c.kind in ("slate", "fork"):
        st.parent = torch.tensor([-1] * c.S + [s for s in range(c.S) for _ in range(c.C)],
                                 dtype=torch.int32, device="cuda")
    if c.kind in ("fork", "compact"):
        st.meta = st.c.meta.clone()   # the tables that every pass starts from
        st.used = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:   # the handle that a user's program keeps, over the same buffers
        from paper_2506_02267_amd import tav2
        t = st.c
        st.cache = tav2.KvCache(k=t.k, v=t.v, k_scale=t.k_scale, v_scale=t.v_scale,
                                k_tail=t.k_tail, v_tail=t.v_tail, table=t.table, length=t.length,
                                fresh=t.fresh, refs=t.refs, max_len=t.max_len)
        st.ws = tav2.Workspace()
    return st


# ------------------------------------------------------------------------- the plain forms
def _row_of(offset, total):
    """(sequence, place in it) of each packed row."""
    r = torch.arange(total, device="cuda")
    s = torch.searchsorted(offset, r, right=True) - 1
    return s, r - offset[s]


def _softmax_v(s, see, v):
    """softmax over the seen keys, the weighted sum of v, log of the sum; nothing seen: 0, -inf."""
    s = s.masked_fill(~see, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l > 0, l, torch.ones_like(l))
    return o, (m + torch.log(l))[..., 0]


def _seen(pos, key, length, window, sinks):
    see = (key <= pos) & (key < length)
    return see & ((pos - key < window) | (key < sinks)) if window else see


def plain_window(st):
    c, G = st.case, st.case.heads // st.case.kv_heads
    total, R, L = st.q.shape[0], c.R, c.L
    p = torch.arange(L, device="cuda")
    rows = (st.offset[:, None] + p).clamp(max=total - 1)
    q = st.q.float()[rows].view(R, L, c.kv_heads, G, c.D).permute(0, 2, 3, 1, 4)
    k = st.k.float()[rows].permute(0, 2, 3, 1).unsqueeze(2).contiguous()
    v = st.v.float()[rows].permute(0, 2, 1, 3).unsqueeze(2).contiguous()
    see = _seen(p[:, None], p, st.length[:, None, None], c.window, c.sinks)[:, None, None]
    o, lse = _softmax_v(torch.matmul(q, k) / math.sqrt(c.D), see, v)
    o = o.permute(0, 3, 1, 2, 4).reshape(R, L, c.heads, c.D)
    lse = lse.permute(0, 3, 1, 2).reshape(R, L, c.heads)
    s, i = _row_of(st.offset, total)
    st.out.copy_(o[s, i])
    st.lse.copy_(lse[s, i])
    return {"out": st.out, "lse": st.lse}


def plain_attend(st, mask, window, sinks, layer=0):
    c, t = st.case, st.c
    H, G, D = c.kv_heads, c.heads // c.kv_heads, c.D
    S, total, n = t.length.shape[0], st.q.shape[0], st.n
    B = t.table.shape[1]
    length = t.length.long()
    page = t.table.long().clamp(min=0)
    block = torch.arange(B, device="cuda")
    open_ = (block == (length // P)[:, None])[:, :, None, None, None]
    k = t.k[layer][page].float() * t.k_scale[layer][page][..., None, None]
    k = torch.where(open_, t.k_tail[layer].float()[:, None], k)              # [S, B, H, P, D]
    v = t.v[layer][page].float() * t.v_scale[layer][page][..., None, None]
    v = torch.where(open_, t.v_tail[layer].float()[:, None], v)              # [S, B, H, D, P]
    k = k.permute(0, 2, 4, 1, 3).reshape(S, H, D, B * P)
    v = v.permute(0, 2, 1, 4, 3).reshape(S, H, B * P, D)
    count = st.offset[1:] - st.offset[:-1]
    i = torch.arange(n, device="cuda")
    rows = (st.offset[:-1, None] + i).clamp(max=total - 1)
    q = st.q.float()[rows].view(S, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, n * G, D)
    pos = (length - count)[:, None] + i if mask == CAUSAL else length[:, None].expand(S, n)
    key = torch.arange(B * P, device="cuda")
    see = _seen(pos[:, :, None], key, length[:, None, None], window, sinks)   # [S, n, keys]
    held = (t.table >= 0) | (block == (length // P)[:, None])
    see = see & held.repeat_interleave(P, 1)[:, None]
    see = see.repeat_interleave(G, 1)[:, None]
    o, lse = _softmax_v(torch.matmul(q, k) / math.sqrt(D), see, v)
    s, j = _row_of(st.offset, total)
    st.out.copy_(o.view(S, H, n, G, D)[s, :, j].reshape(total, c.heads, D))
    st.lse.copy_(lse.view(S, H, n, G)[s, :, j].reshape(total, c.heads))
    return {"out": st.out, "lse": st.lse}


def plain_extend(t, count):
    """New tokens' pages: the lowest free ones, in the order of the sequences; from the first
    sequence that they do not suffice for on, none is extended."""
    B = t.table.shape[1]
    old, new = t.length // P, (t.length + count) // P
    fits = (count > 0) & (new <= B)
    need = torch.where(fits, new - old, torch.zeros_like(old)).long()
    upto = need.cumsum(0)
    free = t.refs == 0
    granted = fits & (upto <= free.sum())
    got = torch.where(granted, need, torch.zeros_like(need))
    ids = torch.argsort((~free).to(torch.int8), stable=True)
    block = torch.arange(B, device="cuda")
    mine = granted[:, None] & (block >= old[:, None]) & (block < new[:, None])
    rank = (upto - need)[:, None] + block - old[:, None]
    t.table.copy_(torch.where(mine, ids[rank.clamp(0, ids.numel() - 1)].int(), t.table))
    t.refs.add_(((free.long().cumsum(0) <= got.sum()) & free).int())
    t.fresh.copy_(torch.where(granted, count, torch.zeros_like(count)))
    t.length.add_(t.fresh)


def plain_append(t, k, v, offset, most, layer=0):
    """The new tokens' rows: full blocks into their pages in 8 bits, the rest into the tail."""
    S = t.length.shape[0]
    new, fresh = t.length.long(), t.fresh.long()
    old = new - fresh
    block = (old // P)[:, None] + torch.arange(most // P + 2, device="cuda")
    pos = block[:, :, None] * P + torch.arange(P, device="cuda")
    row = (offset[:-1, None, None] + pos - old[:, None, None]).clamp(0, k.shape[0] - 1)
    late = (pos >= old[:, None, None])[..., None, None]
    s = torch.arange(S, device="cuda")
    full = (block < (new // P)[:, None]) & (fresh > 0)[:, None]
    last = (new // P - old // P).clamp(max=block.shape[1] - 1)
    at = torch.arange(P, device="cuda")
    write = ((at < (new % P)[:, None]) & (at >= torch.where(last == 0, old % P, 0 * old)[:, None])
             & (fresh > 0)[:, None])
    ids = t.table.long().gather(1, block.clamp(max=t.table.shape[1] - 1))[full]

    def put(x, tail, pool, scale, by_feature):
        rows = torch.where(late, x[row].float(), tail.float()[:, None])     # [S, NB, P, H, D]
        codes, sc = _quantise(rows[full].transpose(1, 2))
        pool[ids] = codes.transpose(2, 3) if by_feature else codes
        scale[ids] = sc
        return torch.where(write[..., None, None], rows[s, last], tail.float()).to(tail.dtype)

    kt = t.k_tail[layer].transpose(1, 2)
    vt = t.v_tail[layer].permute(0, 3, 1, 2)
    kt.copy_(put(k, kt, t.k[layer], t.k_scale[layer], False))
    vt.copy_(put(v, vt, t.v[layer], t.v_scale[layer], True))


def _count_refs(t, table, sign):
    t.refs.index_add_(0, table.reshape(-1).clamp(min=0).long(),
                      (table.reshape(-1) >= 0).int() * sign)


def plain_fork(t, parent):
    p = parent.long().clamp(min=0)
    ok = (parent >= 0) & (t.length == 0) & (parent[p] < 0)
    table = torch.where(ok[:, None], t.table[p], t.table)
    _count_refs(t, torch.where(ok[:, None], table, torch.full_like(table, -1)), 1)
    t.table.copy_(table)
    t.length.copy_(torch.where(ok, t.length[p], t.length))
    t.fresh.copy_(torch.where(ok, torch.zeros_like(t.fresh), t.fresh))
    held = (torch.arange(P, device="cuda") < (t.length % P)[:, None]) & ok[:, None]
    t.k_tail.copy_(torch.where(held[:, None, :, None], t.k_tail[:, p], t.k_tail))
    t.v_tail.copy_(torch.where(held[:, None, None, :], t.v_tail[:, p], t.v_tail))


def plain_free(t, drop):
    gone = (drop != 0)[:, None]
    _count_refs(t, torch.where(gone, t.table, torch.full_like(t.table, -1)), -1)
    t.table.masked_fill_(gone, -1)
    t.length.masked_fill_(gone[:, 0], 0)
    t.fresh.masked_fill_(gone[:, 0], 0)


def plain_trim(t, window, sinks):
    first = torch.arange(t.table.shape[1], device="cuda") * P
    gone = (first >= sinks) & (first + P <= (t.length - window + 1)[:, None])
    _count_refs(t, torch.where(gone, t.table, torch.full_like(t.table, -1)), -1)
    t.table.masked_fill_(gone, -1)


def plain_compact(t, used):
    held = t.refs > 0
    n = held.sum()
    i = torch.arange(t.refs.shape[0], device="cuda")
    hole, mover = ~held & (i < n), held & (i >= n)
    src = torch.nonzero(mover)[:, 0]
    dst = torch.nonzero(hole)[:, 0]
    t.k[:, dst], t.v[:, dst] = t.k[:, src], t.v[:, src]
    t.k_scale[:, dst], t.v_scale[:, dst] = t.k_scale[:, src], t.v_scale[:, src]
    to = i.clone()
    to[src] = dst
    t.refs[dst] = t.refs[src]
    t.refs[src] = 0
    t.table.copy_(torch.where(t.table >= 0, to[t.table.long().clamp(min=0)].int(), t.table))
    used.copy_(n)


# ------------------------------------------------------------------------- one pass
def _written(t):
    """What kv_append wrote beside the codes: the scales and the open blocks."""
    return {"k_scale": t.k_scale, "v_scale": t.v_scale, "k_tail": t.k_tail, "v_tail": t.v_tail}


def run(st):
    c = st.case
    if own:
        return _run_own(st)
    if c.kind == "window":
        return plain_window(st)
    if c.kind == "attend":
        return plain_attend(st, c.mask, c.window, c.sinks)
    t = st.c
    if c.kind == "ingest":
        plain_extend(t, st.count)
        plain_append(t, st.k, st.v, st.new_offset, st.new_max)
        r = plain_attend(st, NONE, 0, 0)
        plain_free(t, st.drop)
        return {**r, **_written(t)}
    if c.kind == "slate":
        plain_fork(t, st.parent)
        plain_extend(t, st.count)
        plain_append(t, st.k, st.v, st.new_offset, st.new_max)
        r = plain_attend(st, CAUSAL, c.window, c.sinks)
        plain_free(t, st.drop)
        return {**r, **_written(t)}
    t.meta.copy_(st.meta)
    if c.kind == "fork":
        plain_fork(t, st.parent)
        plain_trim(t, c.window, c.sinks)
        return {"meta": t.meta, "k_tail": t.k_tail, "v_tail": t.v_tail}
    plain_compact(t, st.used)
    return {"meta": t.meta, "used": st.used, "k": t.k, "v": t.v, "k_scale": t.k_scale,
            "v_scale": t.v_scale}


def _run_own(st):
    from paper_2506_02267_amd import tav2
    c = st.case
    if c.kind == "window":
        tav2.attend_window(st.q, st.k, st.v, st.offset, st.length, c.L, window=c.window,
                           sinks=c.sinks, out=st.out, lse=st.lse)
        return {"out": st.out, "lse": st.lse}
    x = st.cache
    if c.kind in ("attend", "ingest", "slate"):
        mask, window, sinks = NONE, 0, 0
        if c.kind == "attend":
            mask, window, sinks = c.mask, c.window, c.sinks
        else:
            if c.kind == "slate":
                mask, window, sinks = CAUSAL, c.window, c.sinks
                tav2.kv_fork(x, st.parent)
            tav2.kv_extend(x, st.count)
            tav2.kv_append(x, 0, st.k, st.v, st.new_offset, st.new_max)
        tav2.kv_attend(x, 0, st.q, st.offset, st.n, out=st.out, lse=st.lse, flags=mask,
                       window=window, sinks=sinks, ws=st.ws)
        if c.kind == "attend":
            return {"out": st.out, "lse": st.lse}
        tav2.kv_free(x, st.drop)
        return {"out": st.out, "lse": st.lse, **_written(st.c)}
    t = st.c
    t.meta.copy_(st.meta)
    if c.kind == "fork":
        tav2.kv_fork(x, st.parent)
        tav2.kv_trim(x, c.window, c.sinks)
        return {"meta": t.meta, "k_tail": t.k_tail, "v_tail": t.v_tail}
    tav2.kv_compact(x, st.used, ws=st.ws)
    return {"meta": t.meta, "used": st.used, "k": t.k, "v": t.v, "k_scale": t.k_scale,
            "v_scale": t.v_scale}


# ------------------------------------------------------------------------- in 64 bits
def _exact_rows(q, k, v, first, step, window, sinks):
    """Queries [n, H, D] at positions first + step * i over keys [L, Hkv, D], head by head in
    chunks of rows."""
    n, H, D = q.shape
    L, G = k.shape[0], H // k.shape[1]
    out = torch.zeros(n, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((n, H), -math.inf, dtype=torch.float64, device="cuda")
    j = torch.arange(L, device="cuda")
    for h in range(H):
        kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
        for a in range(0, n, 2048):
            b = min(n, a + 2048)
            pos = first + step * torch.arange(a, b, device="cuda")[:, None]
            seen = j <= pos
            if window:
                seen = seen & ((j > pos - window) | (j < sinks))
            x = (q[a:b, h] @ kh.T) * D ** -0.5
            z = torch.logsumexp(torch.where(seen, x, -math.inf), 1)
            some = torch.isfinite(z)[:, None]
            w = torch.where(seen & some, torch.exp(x - torch.where(some, z[:, None], 0.0)), 0.0)
            out[a:b, h], lse[a:b, h] = w @ vh, z
    return out, lse


def _exact_block(x):
    """What a full block [P, H, D] of tokens stands for in the cache."""
    top = x.abs().amax((0, 2), keepdim=True)
    safe = torch.where(top < TINY, torch.ones_like(top), top)
    return torch.where(top < TINY, torch.zeros_like(x), torch.round(127 * x / safe) * (safe / 127))


def exact(case, seed):
    c = SimpleNamespace(**case)
    if c.kind in ("fork", "compact"):
        return None   # these move and count; nothing is computed
    st = prepare(case, seed)
    outs = []
    if c.kind == "window":
        lens = spread(c.L_min, c.L, c.R)
        if 6.0 * c.D * c.heads * sum(L * L for L in lens) > 2e13:
            return None
        at = 0
        for L in lens:
            q, k, v = (x[at:at + L].double() for x in (st.q, st.k, st.v))
            outs.append(_exact_rows(q, k, v, 0, 1, c.window, c.sinks))
            at += L
    else:
        t, lens = st.c, spread(c.L_min, c.L, c.S)

        def held(s):   # keys and values of resident sequence s [L, H, D]
            L, ids = lens[s], t.table[s, :lens[s] // P].long()
            k = (t.k[0, ids].double() * t.k_scale[0, ids].double()[..., None, None]).transpose(1, 2)
            v = (t.v[0, ids].double() * t.v_scale[0, ids].double()[..., None, None]).permute(0, 3, 1, 2)
            kt = t.k_tail[0, s, :, :L % P].double().transpose(0, 1)
            vt = t.v_tail[0, s, :, :, :L % P].double().permute(2, 0, 1)
            shape = (-1, c.kv_heads, c.D)
            return torch.cat([k.reshape(shape), kt]), torch.cat([v.reshape(shape), vt])

        def joined(x, old, new):   # tokens old.. of x are new: the blocks they fill are quantised
            for a in range(old // P * P, new // P * P, P):
                x[a:a + P] = _exact_block(x[a:a + P])
            return x

        off = st.offset.tolist()
        window, sinks = getattr(c, "window", 0), getattr(c, "sinks", 0)
        for s in range(len(off) - 1):
            if off[s + 1] == off[s]:
                continue
            q = st.q[off[s]:off[s + 1]].double()
            n = q.shape[0]
            if c.kind == "attend":
                k, v = held(s)
                mask = c.mask
            elif c.kind == "ingest":
                a = int(st.new_offset[s])
                k, v = (joined(x[a:a + lens[s]].double(), 0, lens[s]) for x in (st.k, st.v))
                mask = NONE
            else:
                p = int(st.parent[s])
                a = int(st.new_offset[s])
                old, new = lens[p], lens[p] + c.m
                k, v = (joined(torch.cat([h, x[a:a + c.m].double()]), old, new)
                        for h, x in zip(held(p), (st.k, st.v)))
                mask = CAUSAL
            L = k.shape[0]
            outs.append(_exact_rows(q, k, v, L - n if mask == CAUSAL else L,
                                    1 if mask == CAUSAL else 0, window, sinks))
    return {"out": torch.cat([o for o, _ in outs]), "lse": torch.cat([z for _, z in outs])}
