"""The performance cases of a beam search over resident histories: the selection of beams over a
vocabulary (`beam_select`), the reordering of the cache's sequences that follows it (`kv_reorder`) and
the attention of many continuations to the one history that they share (`kv_attend_prefix`).

A case's `kind`:
  select   beam_select: R requests of B beams, a vocabulary of V tokens
  reorder  kv_reorder on restored page tables: surviving beams stay, the others become copies of them
  attend   kv_attend_prefix: the members of U groups over their histories and their own tokens
  step     kv_reorder + kv_extend + kv_append + kv_attend_prefix + beam_select: one step of the search

Where `own` is false, run() computes the same in elementary torch operations on the same buffers: in 32
bits, the values that beams are ranked by in 64.  Histories have the lengths of this repository's
workloads (1024 to 16384 actions, heads of 32 to 128 features), spread evenly over a case's range.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

P = 64                 # tokens of a page
TINY = 2.0 ** -100     # a block below this is stored as zeros
NONE, CAUSAL = 1, 0    # masks, as the library's flags
LOWEST = -torch.finfo(torch.float32).max


# ------------------------------------------------------------------------- cases
def _named(name, c):
    return dict(c, name=name) if name else c


def _select(name, dtype, R, B, V, keep, pad=0, ended=0.0, mask="", place=False):
    """`pad`: elements between rows; `ended`: share of finished beams; `mask`: tokens allowed for every
    beam ("all") or for each ("row"); `place`: surviving beams keep their places."""
    return _named(name, dict(kind="select", dtype=dtype, R=R, B=B, V=V, keep=keep, pad=pad,
                             ended=ended, mask=mask, place=place))


def _reorder(name, U, B_min, B, own_min, own_max, layers, kv_heads, D, moved):
    """`moved`: share of the members that become copies of another."""
    return _named(name, dict(kind="reorder", U=U, B_min=B_min, B=B, own_min=own_min, own_max=own_max,
                             layers=layers, kv_heads=kv_heads, D=D, moved=moved))


def _attend(name, U, L_min, L, B_min, B, own_min, own_max, n_min, n, heads, kv_heads, D, mask=CAUSAL,
            window=0, sinks=0):
    """U histories of L_min .. L tokens, B_min .. B members each with own_min .. own_max tokens of their
    own and n_min .. n queries."""
    return _named(name, dict(kind="attend", U=U, L_min=L_min, L=L, B_min=B_min, B=B, own_min=own_min,
                             own_max=own_max, n_min=n_min, n=n, heads=heads, kv_heads=kv_heads, D=D,
                             mask=mask, window=window, sinks=sinks))


def _step(name, U, L_min, L, B, own_min, own_max, heads, kv_heads, D, V, moved):
    return _named(name, dict(kind="step", U=U, L_min=L_min, L=L, B_min=B, B=B, own_min=own_min,
                             own_max=own_max, n_min=1, n=1, heads=heads, kv_heads=kv_heads, D=D, V=V,
                             mask=CAUSAL, window=0, sinks=0, moved=moved, layers=1))


def listed():
    return [
        # one user, 8 beams, items as codes of 256 values: the smallest call, latency
        _select("select_one", "bf16", 1, 8, 256, 8),
        # 256 users, 32 beams, a codebook of 4096, some beams finished, survivors in place
        _select("select_codes", "bf16", 256, 32, 4096, 32, ended=0.1, place=True),
        # a catalogue of items as one vocabulary of odd size, fp32, tokens allowed for each beam
        _select("select_items", "f32", 16, 16, 100003, 50, pad=3, mask="row"),
        # a batch over a large vocabulary: the largest selection
        _select("select_large", "bf16", 32, 32, 131072, 32),
        # one user's beams early in the search: latency
        _reorder("reorder_one", 1, 8, 8, 3, 3, 4, 4, 64, 0.5),
        # 64 users, continuations of up to 200 tokens, 8 layers
        _reorder("reorder_batch", 64, 20, 32, 1, 200, 8, 4, 64, 0.5),
        # one user, 8 beams over a history of 16384: latency
        _attend("attend_one", 1, 16384, 16384, 8, 8, 3, 3, 1, 1, 4, 4, 64),
        # 64 users, 16 beams each, shared key heads
        _attend("attend_beams", 64, 1024, 16384, 16, 16, 1, 20, 1, 1, 8, 2, 64),
        # few users with many continuations each, wide heads, a window
        _attend("attend_window", 12, 700, 16384, 3, 64, 2, 90, 1, 1, 8, 4, 128, CAUSAL, 2000, 7),
        # branches of several tokens at once (drafts, slates), own tokens beyond a page
        _attend("attend_branches", 16, 1024, 16384, 8, 8, 6, 150, 1, 6, 4, 4, 64),
        # a whole step for 16 users of 16 beams
        _step("step", 16, 1024, 16384, 16, 2, 62, 8, 2, 64, 4096, 0.5),
        # and for one user: latency
        _step("step_one", 1, 4096, 4096, 8, 4, 4, 4, 4, 64, 1024, 0.4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["select", "select", "select", "reorder", "attend", "attend", "attend", "step"])
    if kind == "select":
        B = _log(rng, 1, 100)
        V = _log(rng, 40, 131072)
        R = _log(rng, 1, max(1, min(256, int(1.2e8 / (B * V)))))
        place = rng.random() < 0.3
        keep = B if place else min(_log(rng, 1, 100), B * V)
        return _select(None, rng.choice(["bf16", "bf16", "f32"]), R, B, V, keep,
                       rng.choice([0, 0, rng.randint(1, 40)]), rng.choice([0.0, 0.0, 0.2]),
                       rng.choice(["", "", "all", "row"]), place)
    D = rng.choice([32, 64, 64, 128])
    kv_heads = rng.choice([1, 2, 4])
    B = _log(rng, 2, 64)
    if kind == "reorder":
        U = _log(rng, 1, max(1, min(64, 2000 // B)))
        most = _log(rng, 1, 300)
        return _reorder(None, U, rng.randint(1, B), B, rng.randint(0, most), most,
                        rng.randint(1, 8 if D < 128 else 4), kv_heads, D, rng.uniform(0.1, 0.9))
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    low = rng.choice([1.0, 0.5, 0.06])
    L = _log(rng, 20, 16384)
    n = rng.choice([1, 1, rng.randint(2, 8)])
    U = _log(rng, 1, max(1, min(64, int(1.5e8 / (L * B * n * heads) * min(1.0, 64 / D)))))
    if kind == "step":
        most = rng.randint(1, 90)
        return _step(None, U, max(1, int(L * low)), L, B, rng.randint(0, most), most, heads, kv_heads, D,
                     _log(rng, max(40, B), 5000), rng.uniform(0.1, 0.9))
    mask = rng.choice([CAUSAL, CAUSAL, NONE])
    window = rng.choice([0, 0, _log(rng, 1, 4000)])
    most = n + _log(rng, 1, 200)
    return _attend(None, U, max(1, int(L * low)), L, rng.randint(1, B), B, rng.randint(n, most), most,
                   rng.choice([1, n]), n, heads, kv_heads, D, mask, window,
                   rng.choice([0, 4, 70]) if window else 0)


def spread(lo, hi, n):
    """n whole numbers spread evenly over lo..hi, in an order of no pattern."""
    v = [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(n * 1000003 + hi).shuffle(v)
    return v


def _sizes(c):
    """(histories' lengths, members of each group, members' own lengths, their queries)."""
    members = spread(c.B_min, c.B, c.U)
    m = sum(members)
    lens = spread(c.L_min, c.L, c.U) if hasattr(c, "L") else []
    return lens, members, spread(c.own_min, c.own_max, m), spread(getattr(c, "n_min", 0),
                                                                  getattr(c, "n", 0), m)


def _parents(members, moved, seed):
    """The member that each one continues (an index in its group): those that go on stay where they
    are, about `moved` of them become copies of one that does."""
    r = random.Random(seed)
    out = []
    for n in members:
        gone = r.sample(range(n), min(n - 1, round(moved * n)))
        stay = [i for i in range(n) if i not in set(gone)]
        out += [r.choice(stay) if i in set(gone) else i for i in range(n)]
    return out


# ------------------------------------------------------------------------- work
def _attend_work(c, lens, members, owns, counts):
    """Bytes and operations of the attention: a history's keys that some query sees, once a group."""
    keys = pairs = rows = m = 0
    for L, b in zip(lens, members):
        first = L
        for own_len, n in zip(owns[m:m + b], counts[m:m + b]):
            rows += n
            keys += own_len
            for i in range(n):
                o = own_len - n + i if c.mask == CAUSAL else own_len   # the query's place behind the history
                low = max(0, L + o - c.window + 1) if c.window else 0
                pairs += max(0, L - low) + min(c.sinks, low, L)
                pairs += min(own_len, o + 1) - max(0, min(own_len, low - L))
                first = min(first, low)
        keys += L - first + min(c.sinks, first)
        m += b
    return {"bytes": keys * c.kv_heads * (2 * c.D + 8 / P) + rows * c.heads * (4 * c.D + 4),
            "flops": 4.0 * c.D * c.heads * pairs}


def _reorder_work(c, members, owns, parents):
    moved = [owns[first + p] for first, i, p in _members(members, parents) if p != i]
    tails = sum(n % P for n in moved) * 2 * c.kv_heads * c.D * 2 * c.layers
    return {"bytes": 2 * tails + sum(n // P for n in moved) * 24 + sum(members) * 8, "flops": 0}


def _members(members, parents):
    at = 0
    for n in members:
        for i in range(n):
            yield at, i, parents[at + i]
        at += n


def _select_work(rows, V, es, keep, mask):
    return {"bytes": rows * V * (es + (0.125 if mask == "row" else 0.0)) + rows * 5 + keep * 13,
            "flops": 4.0 * rows * V}


def work(case):
    c = SimpleNamespace(**case)
    if c.kind == "select":
        return _select_work(c.R * c.B, c.V, 2 if c.dtype == "bf16" else 4, c.R * c.keep, c.mask)
    lens, members, owns, counts = _sizes(c)
    if c.kind == "attend":
        return _attend_work(c, lens, members, owns, counts)
    parents = _parents(members, c.moved, 1)
    if c.kind == "reorder":
        return _reorder_work(c, members, owns, parents)
    a = _attend_work(c, lens, members, [n + 1 for n in owns], counts)
    r = _reorder_work(c, members, owns, parents)
    s = _select_work(c.U * c.B, c.V, 2, c.U * c.B, "")
    new = sum(members) * 2 * c.kv_heads * c.D * 4
    return {"bytes": a["bytes"] + r["bytes"] + s["bytes"] + new, "flops": a["flops"] + s["flops"]}


# ------------------------------------------------------------------------- inputs
def _quantise(x):
    """(codes int8, scale) of x [..., P, D]: one scale for the last two axes."""
    top = x.abs().amax((-2, -1), keepdim=True)
    small = top < TINY
    top = torch.where(small, torch.full_like(top, 127.0), top)
    n = torch.full_like(top, 127.0)
    codes = torch.round(x * n / top).clamp(-127, 127)
    codes = torch.where(small, torch.zeros_like(codes), codes)
    return codes.to(torch.int8), (top / n)[..., 0, 0]


def _cache(g, layers, pages, seqs, kv_heads, D, max_blocks, meta):
    """A cache's buffers; pages and tails hold random tokens (values wider in some features than in
    others, as projections give)."""
    dev = "cuda"
    shape = (layers, pages, kv_heads, P, D)
    t = SimpleNamespace(
        k=torch.zeros(shape, dtype=torch.int8, device=dev),
        v=torch.zeros(layers, pages, kv_heads, D, P, dtype=torch.int8, device=dev),
        k_scale=torch.ones(layers, pages, kv_heads, device=dev),
        v_scale=torch.ones(layers, pages, kv_heads, device=dev),
        k_tail=torch.zeros(layers, seqs, kv_heads, P, D, dtype=torch.bfloat16, device=dev),
        v_tail=torch.zeros(layers, seqs, kv_heads, D, P, dtype=torch.bfloat16, device=dev))
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


def _tables(lens, max_blocks, pages, seed):
    """[table | length | fresh | refs]: sequences of `lens` tokens on pages that lie anywhere in the pool."""
    r = torch.Generator().manual_seed(seed)
    ids = torch.randperm(pages, generator=r)
    seqs = len(lens)
    table = torch.full((seqs, max_blocks), -1, dtype=torch.int64)
    refs = torch.zeros(pages, dtype=torch.int64)
    at = 0
    for s, L in enumerate(lens):
        n = L // P
        table[s, :n] = ids[at:at + n]
        at += n
    refs[ids[:at]] = 1
    return torch.cat([table.view(-1), torch.tensor(lens), torch.zeros(seqs, dtype=torch.int64), refs])


def _offsets(counts, dtype=torch.int64):
    o = [0]
    for n in counts:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=dtype, device="cuda"), o[-1]


def _rows(g, n, heads, D):
    return torch.randn(n, heads, D, generator=g, device="cuda").to(torch.bfloat16)


def _prepare_select(st, g, R, B, V, keep, dtype, pad, ended, mask):
    """Logits as a model gives them: what a request's beams agree on and what is each one's own; beams
    that have come as far as some unlikely tokens."""
    dev = "cuda"
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    st.logits = torch.empty(R * B, V + pad, dtype=dt, device=dev)[:, :V]
    for r in range(R):
        shared = 1.5 * torch.randn(1, V, generator=g, device=dev)
        st.logits[r * B:(r + 1) * B] = shared + 1.5 * torch.randn(B, V, generator=g, device=dev)
    st.score = -8.0 * torch.rand(R, B, generator=g, device=dev)
    st.done = (torch.rand(R, B, generator=g, device=dev) < ended).to(torch.uint8)
    st.allowed = None
    if mask:
        st.allowed = torch.randint(0, 256, (R * B if mask == "row" else 1, (V + 7) // 8), generator=g,
                                   device=dev, dtype=torch.uint8)
    st.eos = min(2, V - 1)
    st.beams, st.keep = B, keep
    st.parent = torch.empty(R, keep, dtype=torch.int32, device=dev)
    st.token = torch.empty(R, keep, dtype=torch.int32, device=dev)
    st.best = torch.empty(R, keep, device=dev)
    st.ends = torch.empty(R, keep, dtype=torch.uint8, device=dev)


def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = SimpleNamespace(case=c)
    if c.kind == "select":
        _prepare_select(st, g, c.R, c.B, c.V, c.keep, c.dtype, c.pad, c.ended, c.mask)
        st.place = c.place
    else:
        lens, members, owns, counts = _sizes(c)
        layers, M = getattr(c, "layers", 1), sum(members)
        first = len(lens)   # the histories come first, the members behind them
        seqs = first + M
        pages = sum(n // P for n in lens + owns) + 7 + (M if c.kind == "step" else 0)
        blocks = max(lens + owns) // P + 3
        meta = _tables(lens + owns, blocks, pages, seed)
        st.c = _cache(g, layers, pages, seqs, c.kv_heads, c.D, blocks, meta)
        st.c.max_len = max(lens + owns) + 1
        st.group, _ = _offsets(members, torch.int32)
        st.group += first
        st.prefix = torch.arange(first, dtype=torch.int32, device="cuda") if first else None
        st.first, st.members = first, max(members)
        st.own_most = max(owns) + (1 if c.kind == "step" else 0)
        if c.kind in ("reorder", "step"):
            st.order = torch.tensor(_parents(members, c.moved, seed), dtype=torch.int32, device="cuda")
            st.meta = st.c.meta.clone()   # the tables that every pass starts from
        if c.kind in ("attend", "step"):
            st.offset, total = _offsets([0] * first + counts)
            st.n = max(counts)
            st.q = _rows(g, total, c.heads, c.D) * 1.5
            st.out = torch.empty(total, c.heads, c.D, dtype=torch.bfloat16, device="cuda")
            st.lse = torch.empty(total, c.heads, device="cuda")
        if c.kind == "step":
            st.count = torch.tensor([0] * first + [1] * M, dtype=torch.int32, device="cuda")
            st.k, st.v = _rows(g, M, 2 * c.kv_heads, c.D).split([c.kv_heads, c.kv_heads], 1)
            _prepare_select(st, g, c.U, c.B, c.V, c.B, "bf16", 0, 0.0, "")
            st.place = True
    if own:   # the handles that a user's program keeps, over the same buffers
        from paper_2506_02267_amd import tav2
        if c.kind != "select":
            t = st.c
            st.cache = tav2.KvCache(k=t.k, v=t.v, k_scale=t.k_scale, v_scale=t.v_scale,
                                    k_tail=t.k_tail, v_tail=t.v_tail, table=t.table, length=t.length,
                                    fresh=t.fresh, refs=t.refs, max_len=t.max_len)
            st.groups = tav2.KvGroups(st.group, st.prefix, max_members=st.members,
                                      max_own=st.own_most)
        st.ws = tav2.Workspace()
    return st


# ------------------------------------------------------------------------- the plain forms
def plain_select(st):
    """The `keep` best continuations of every request's beams, best first; equal ones: the lower beam
    first, then the lower token."""
    B, K = st.beams, st.keep
    R, V = st.score.shape[0], st.logits.shape[1]
    z = st.logits.double().view(R, B, V)
    there = torch.isfinite(z)
    top = torch.where(there, z, torch.full_like(z, -1e300)).amax(-1, keepdim=True)
    total = torch.where(there, torch.exp(z - top), torch.zeros_like(z)).sum(-1, keepdim=True)
    base = st.score.double()[..., None] - (top + torch.log(total))
    value = base + z
    live = torch.isfinite(st.score)[..., None]
    ended = (st.done != 0)[..., None]
    is_candidate = there & live & ~ended
    if st.allowed is not None:
        v = torch.arange(V, device="cuda")
        bits = (st.allowed[:, v // 8] >> (v % 8).to(torch.uint8)) & 1
        is_candidate &= (bits != 0).view(-1, B, V) if bits.shape[0] > 1 else (bits != 0)
    value = torch.where(is_candidate, value, torch.full_like(value, -math.inf))
    # a finished beam goes on as itself
    itself = live & ended & (torch.arange(V, device="cuda") == st.eos)
    value = torch.where(itself, st.score.double()[..., None], value).view(R, B * V)
    del z, there, is_candidate, itself
    kth = torch.topk(value, K, dim=1).values[:, -1:]
    kept = (value >= kth) & (value > -math.inf)
    r, at = torch.nonzero(kept, as_tuple=True)   # by request, beam and token
    best = value[r, at]
    order = torch.argsort(best, descending=True, stable=True)
    order = order[torch.argsort(r[order], stable=True)]
    r, at, best = r[order], at[order], best[order]
    count = kept.sum(1)
    place = torch.arange(r.shape[0], device="cuda") - (count.cumsum(0) - count)[r]
    st.parent.fill_(-1)
    st.token.fill_(-1)
    st.best.fill_(-math.inf)
    st.ends.fill_(0)
    r, at, best, place = (x[place < K] for x in (r, at, best, place))
    parent = at // V
    if st.place:   # a beam's best continuation stays in its place, the others take the free ones
        rank = torch.full((R, B), -1, device="cuda", dtype=torch.long)
        rank[r, place] = parent
        i = torch.arange(B, device="cuda")
        earlier = (rank[:, :, None] == rank[:, None, :]) & (i[None, :] < i[:, None])
        heads_it = (rank >= 0) & ~earlier.any(-1)
        taken = (heads_it[:, :, None] & (rank[:, :, None] == i)).any(1)
        free = torch.argsort(taken.to(torch.int8), dim=1, stable=True)   # free places first
        nth = (~heads_it).long().cumsum(1) - 1
        slot = torch.where(heads_it, rank, free.gather(1, nth.clamp(min=0)))
        place = slot[r, place]
    st.parent[r, place] = parent.int()
    st.token[r, place] = (at % V).int()
    st.best[r, place] = best.clamp(min=LOWEST).float()
    st.ends[r, place] = ((st.done[r, parent] != 0) | (at % V == st.eos)).to(torch.uint8)
    return {"parent": st.parent, "token": st.token, "score": st.best, "done": st.ends}


def _count_refs(t, table, sign):
    t.refs.index_add_(0, table.reshape(-1).clamp(min=0).long(),
                      (table.reshape(-1) >= 0).int() * sign)


def _source(st):
    """The sequence that each one continues."""
    s = torch.arange(st.c.length.shape[0], device="cuda")
    g = torch.searchsorted(st.group.long(), s, right=True) - 1
    src = s.clone()
    src[st.first:] = st.group.long()[g[st.first:]] + st.order.long()
    return s, src


def plain_reorder(st):
    t = st.c
    s, src = _source(st)
    moved = src != s
    table = torch.where(moved[:, None], t.table[src], t.table)
    _count_refs(t, t.table, -1)
    _count_refs(t, table, 1)
    t.table.copy_(table)
    t.fresh.copy_(torch.where(moved, torch.zeros_like(t.fresh), t.fresh))
    t.length.copy_(t.length[src])
    held = (torch.arange(P, device="cuda") < (t.length % P)[:, None]) & moved[:, None]
    t.k_tail.copy_(torch.where(held[:, None, :, None], t.k_tail[:, src], t.k_tail))
    t.v_tail.copy_(torch.where(held[:, None, None, :], t.v_tail[:, src], t.v_tail))


def plain_extend(t, count):
    """New tokens' pages: the lowest free ones, in the order of the sequences."""
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


def plain_append_one(t, k, v, first):
    """One new token for each sequence from `first` on: into the open block, which goes to its page in 8
    bits once it is full."""
    new = t.length[first:].long()
    at = (new - 1) % P
    s = torch.arange(first, t.length.shape[0], device="cuda")
    full = new % P == 0
    e = ~full
    t.k_tail[0, s[e], :, at[e]] = k[e]
    t.v_tail[0, s[e], :, :, at[e]] = v[e]
    s = s[full]
    ids = t.table[s, new[full] // P - 1].long()
    kb, vb = t.k_tail[0, s].float(), t.v_tail[0, s].float()
    kb[:, :, P - 1], vb[..., P - 1] = k[full].float(), v[full].float()
    t.k[0, ids], t.k_scale[0, ids] = _quantise(kb)
    t.v[0, ids], t.v_scale[0, ids] = _quantise(vb)


def _held(t, layer, seqs, blocks):
    """Keys [n, H, D, blocks * P] and values [n, H, blocks * P, D] of sequences, and which are there."""
    H, D = t.k.shape[2], t.k.shape[4]
    table, length = t.table[seqs, :blocks], t.length[seqs]
    page = table.long().clamp(min=0)
    block = torch.arange(blocks, device="cuda")
    is_open = block == (length // P)[:, None]
    o = is_open[:, :, None, None, None]
    k = t.k[layer][page].float() * t.k_scale[layer][page][..., None, None]
    k = torch.where(o, t.k_tail[layer][seqs].float()[:, None], k)             # [n, B, H, P, D]
    v = t.v[layer][page].float() * t.v_scale[layer][page][..., None, None]
    v = torch.where(o, t.v_tail[layer][seqs].float()[:, None], v)             # [n, B, H, D, P]
    there = ((table >= 0) | is_open).repeat_interleave(P, 1)
    there &= torch.arange(blocks * P, device="cuda") < length[:, None]
    return (k.permute(0, 2, 4, 1, 3).reshape(-1, H, D, blocks * P),
            v.permute(0, 2, 1, 4, 3).reshape(-1, H, blocks * P, D), there)


def plain_attend(st, mask, window, sinks):
    """Each group's queries over its history, each member's over its own tokens, one softmax over both."""
    c, t = st.case, st.c
    H, G, D, U = c.kv_heads, c.heads // c.kv_heads, c.D, st.prefix.shape[0]
    total, n, B = st.q.shape[0], st.n, st.members
    count = (st.offset[1:] - st.offset[:-1])
    seqs = torch.arange(st.first, t.length.shape[0], device="cuda")
    group = torch.searchsorted(st.group.long(), seqs, right=True) - 1
    slot = seqs - st.group.long()[group]
    # the members' queries by (group, member, place)
    i = torch.arange(n, device="cuda")
    rows = torch.zeros(U, B, n, dtype=torch.long, device="cuda")
    rows[group, slot] = (st.offset[seqs][:, None] + i).clamp(max=total - 1)
    own_len = torch.zeros(U, B, dtype=torch.long, device="cuda")
    own_len[group, slot] = t.length[seqs].long()
    asked = torch.zeros(U, B, dtype=torch.long, device="cuda")
    asked[group, slot] = count[seqs]
    place = (own_len - asked)[..., None] + i if mask == CAUSAL else own_len[..., None].expand(U, B, n)
    L = t.length[st.prefix.long()].long()
    pos = L[:, None, None] + place                                            # [U, B, n]
    q = st.q.float()[rows].view(U, B, n, H, G, D) / math.sqrt(D)
    # the history's scores, once a group
    blocks = int(c.L) // P + 1
    k, v, there = _held(t, 0, st.prefix.long(), blocks)
    key = torch.arange(blocks * P, device="cuda")
    see = there[:, None, None].expand(U, B, n, -1)
    if window:
        see = see & ((pos[..., None] - key < window) | (key < sinks))
    qp = q.permute(0, 3, 1, 2, 4, 5).reshape(U, H, B * n * G, D)
    sp = torch.matmul(qp, k).view(U, H, B, n, G, -1)
    sp = sp.masked_fill_(~see[:, None, :, :, None], -math.inf)
    # the own tokens' scores, a member's own
    blocks = int(st.own_most) // P + 1
    ko, vo, there = _held(t, 0, seqs, blocks)
    key = torch.arange(blocks * P, device="cuda")
    gpos, gplace = pos[group, slot], place[group, slot]                       # [M, n]
    see = there[:, None] & (key <= gplace[..., None])
    if window:
        at = L[group][:, None, None] + key
        see &= (gpos[..., None] - at < window) | (at < sinks)
    M = seqs.shape[0]
    qo = q[group, slot].permute(0, 2, 1, 3, 4).reshape(M, H, n * G, D)
    so = torch.matmul(qo, ko).view(M, H, n, G, -1).masked_fill_(~see[:, None, :, None], -math.inf)
    # one softmax over both
    mp = sp.amax(-1)[group, :, slot]                                          # [M, H, n, G]
    m = torch.maximum(mp, so.amax(-1))
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    ref = torch.zeros(U, B, H, n, G, device="cuda")
    ref[group, slot] = m
    sp = sp.sub_(ref.permute(0, 2, 1, 3, 4)[..., None]).exp_()
    op = torch.matmul(sp.view(U, H, B * n * G, -1), v).view(U, H, B, n, G, D)[group, :, slot]
    lp = sp.sum(-1)[group, :, slot]
    so = torch.exp(so - m[..., None])
    o = op + torch.matmul(so.view(M, H, n * G, -1), vo).view(M, H, n, G, D)
    l = lp + so.sum(-1)
    o = (o / torch.where(l > 0, l, torch.ones_like(l))[..., None]).permute(0, 2, 1, 3, 4)
    lse = (m + torch.log(l)).permute(0, 2, 1, 3)
    r = torch.arange(total, device="cuda")
    s = torch.searchsorted(st.offset, r, right=True) - 1
    j, s = r - st.offset[s], s - st.first
    st.out.copy_(o[s, j].reshape(total, c.heads, D))
    st.lse.copy_(lse[s, j].reshape(total, c.heads))
    return {"out": st.out, "lse": st.lse}


# ------------------------------------------------------------------------- one pass
def _state(t):
    """Page tables, lengths and holders, and the open blocks."""
    return {"meta": t.meta, "k_tail": t.k_tail, "v_tail": t.v_tail}


def run(st):
    c = st.case
    if own:
        return _run_own(st)
    if c.kind == "select":
        return plain_select(st)
    if c.kind == "attend":
        return plain_attend(st, c.mask, c.window, c.sinks)
    t = st.c
    t.meta.copy_(st.meta)
    plain_reorder(st)
    if c.kind == "reorder":
        return _state(t)
    plain_extend(t, st.count)
    plain_append_one(t, st.k, st.v, st.first)
    r = plain_attend(st, CAUSAL, 0, 0)
    return {**r, **plain_select(st), **_state(t), "k_scale": t.k_scale, "v_scale": t.v_scale}


def _run_own(st):
    from paper_2506_02267_amd import tav2
    c = st.case

    def select():
        tav2.beam_select(st.logits, st.beams, st.keep, score=st.score, done=st.done,
                         allowed=st.allowed, eos=st.eos,
                         flags=tav2.BEAM_IN_PLACE if st.place else tav2.BEAM_RANKED,
                         out=(st.parent, st.token, st.best, st.ends), ws=st.ws)
        return {"parent": st.parent, "token": st.token, "score": st.best, "done": st.ends}

    def attend(mask, window, sinks):
        tav2.kv_attend_prefix(st.cache, 0, st.groups, st.q, st.offset, st.n, out=st.out, lse=st.lse,
                              flags=mask, window=window, sinks=sinks, ws=st.ws)
        return {"out": st.out, "lse": st.lse}

    if c.kind == "select":
        return select()
    if c.kind == "attend":
        return attend(c.mask, c.window, c.sinks)
    t = st.c
    t.meta.copy_(st.meta)
    tav2.kv_reorder(st.cache, st.groups, st.order)
    if c.kind == "reorder":
        return _state(t)
    tav2.kv_extend(st.cache, st.count)
    tav2.kv_append(st.cache, 0, st.k, st.v, st.offset, 1)
    r = attend(CAUSAL, 0, 0)
    return {**r, **select(), **_state(t), "k_scale": t.k_scale, "v_scale": t.v_scale}


# ------------------------------------------------------------------------- in 64 bits
def _exact_scores(st):
    """The selected values alone, request by request."""
    B, K = st.beams, st.keep
    R, V = st.score.shape[0], st.logits.shape[1]
    out = torch.empty(R, K, dtype=torch.float64, device="cuda")
    for r in range(R):
        lists, beam = [], []
        for b in range(B):
            s = float(st.score[r, b])
            if not math.isfinite(s):
                continue
            if int(st.done[r, b]):
                lists.append(torch.tensor([s], dtype=torch.float64, device="cuda"))
                beam.append(b)
                continue
            z = st.logits[r * B + b].double()
            z = torch.where(torch.isfinite(z), z, torch.full_like(z, -math.inf))
            x = s + torch.log_softmax(z, 0)
            if st.allowed is not None:
                bytes_ = st.allowed[r * B + b if st.allowed.shape[0] > 1 else 0]
                bits = torch.stack([(bytes_ >> e) & 1 for e in range(8)], 1).reshape(-1)[:V]
                x = x[bits != 0]
            lists.append(torch.sort(x, descending=True).values[:K])
            beam += [b] * lists[-1].numel()
        if not lists:
            out[r] = -math.inf
            continue
        x, at = torch.sort(torch.cat(lists), descending=True, stable=True)
        x, at = x[:K].tolist(), at[:K].tolist()
        best = [(v, beam[a]) for v, a in zip(x, at) if math.isfinite(v)]
        places = [None] * K
        if st.place:
            for v, b in best:
                if places[b] is None:
                    places[b] = v
        later, seen = [], set()
        for v, b in best:
            if not st.place or b in seen:
                later.append(v)
            seen.add(b)
        later = iter(later)
        out[r] = torch.tensor([next(later, -math.inf) if v is None else v for v in places],
                              dtype=torch.float64)
    return out


def _exact_block(x):
    """What a full block [P, H, D] of tokens stands for in the cache."""
    top = x.abs().amax((0, 2), keepdim=True)
    safe = torch.where(top < TINY, torch.ones_like(top), top)
    return torch.where(top < TINY, torch.zeros_like(x), torch.round(127 * x / safe) * (safe / 127))


def exact(case, seed):
    c = SimpleNamespace(**case)
    if c.kind == "reorder":
        return None   # this moves and counts; nothing is computed
    st = prepare(case, seed)
    if c.kind == "select":
        return {"parent": None, "token": None, "score": _exact_scores(st), "done": None}
    t = st.c
    lens, members, owns, counts = _sizes(c)
    if 6.0 * c.D * c.heads * sum(L * b for L, b in zip(lens, members)) * c.n > 2e13:
        return None
    shape = (-1, c.kv_heads, c.D)

    def held(s):   # keys and values of sequence s [L, H, D]
        L = (lens + owns)[s]
        ids = t.table[s, :L // P].long()
        k = (t.k[0, ids].double() * t.k_scale[0, ids].double()[..., None, None]).transpose(1, 2)
        v = (t.v[0, ids].double() * t.v_scale[0, ids].double()[..., None, None]).permute(0, 3, 1, 2)
        kt = t.k_tail[0, s, :, :L % P].double().transpose(0, 1)
        vt = t.v_tail[0, s, :, :, :L % P].double().permute(2, 0, 1)
        return torch.cat([k.reshape(shape), kt]), torch.cat([v.reshape(shape), vt])

    outs, lses = [], []
    order = st.order.tolist() if c.kind == "step" else None
    m = 0
    for g, (L, b) in enumerate(zip(lens, members)):
        kp, vp = held(g)
        for j in range(b):
            src = st.first + m + (order[m + j] if order else j)
            k, v = held(src)
            if c.kind == "step":   # the new token, which may fill a block
                k, v = (torch.cat([x, y[m + j].double()[None]]) for x, y in ((k, st.k), (v, st.v)))
                a = k.shape[0] // P * P
                if k.shape[0] == a:
                    k[a - P:], v[a - P:] = _exact_block(k[a - P:]), _exact_block(v[a - P:])
            n = counts[m + j]
            at = int(st.offset[st.first + m + j])
            q = st.q[at:at + n].double()
            i = torch.arange(n, device="cuda")
            o = k.shape[0]
            place = (o - n + i if c.mask == CAUSAL else torch.full_like(i, o))[:, None]
            k, v = torch.cat([kp, k]), torch.cat([vp, v])
            key = torch.arange(L + o, device="cuda")
            see = (key < L) | (key - L <= place)
            if c.window:
                see &= (key > L + place - c.window) | (key < c.sinks)
            out = torch.zeros(n, c.heads, c.D, dtype=torch.float64, device="cuda")
            lse = torch.full((n, c.heads), -math.inf, dtype=torch.float64, device="cuda")
            for h in range(c.kv_heads):
                G = c.heads // c.kv_heads
                kh, vh = k[:, h].contiguous(), v[:, h].contiguous()
                x = (q[:, h * G:(h + 1) * G].reshape(n * G, c.D) @ kh.T) * c.D ** -0.5
                w = see.repeat_interleave(G, 0)
                x = torch.where(w, x, -math.inf)
                z = torch.logsumexp(x, 1)
                some = torch.isfinite(z)[:, None]
                p = torch.where(w & some, torch.exp(x - torch.where(some, z[:, None], 0.0)), 0.0)
                out[:, h * G:(h + 1) * G] = (p @ vh).view(n, G, c.D)
                lse[:, h * G:(h + 1) * G] = z.view(n, G)
            outs.append(out)
            lses.append(lse)
        m += b
    r = {"out": torch.cat(outs), "lse": torch.cat(lses)}
    if c.kind == "step":
        r.update({n: None for n in ("parent", "token", "score", "done", "meta", "k_tail", "v_tail",
                                    "k_scale", "v_scale")})
    return r
