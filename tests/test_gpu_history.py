"""Attention over whole histories on the GPU against the 64-bit oracle (oracle/history.py): the
windowed attention of packed sequences, and the paged 8-bit cache, whose tables, counts and codes are
compared exactly.

Bounds.  A rounding to bf16 is off by at most B = 2^-8 of the value.  An output is a sum of weights
times values, rounded once; its weights are rounded to bf16 once (bf16 path), so with
size = sum of weights times |v|:  |error| <= B |o| + B size + what fp32 adds.  A score's fp32 dot
product of D terms is off by at most d = (D + 4) 2^-24 reach (reach: scale * sum |q k|), and its
exponent's argument by 2^-23 of its magnitude, which reach bounds too; both move a weight by that
relative amount, and the normalising sum again: 2 (d + 2 reach 2^-23) size.  Sums of n weights in
fp32 add at most n 2^-24, exponentials and reciprocals a few 2^-23.

The cache's weights are fp16 (times the values' scale, against a reference that keeps the largest
such product at 2^6 or more): off by at most 2^-11 of the weight, or by half the least step, 2^-25,
which is 2^-31 of the largest product.  A key's code is at most 127, and 127 times the largest
product's scale is at most the largest |v|, so the latter adds at most n 2^-31 max|v|."""
import numpy as np
import pytest
import torch

from oracle import history
from paper_2506_02267_amd import tav2 as T

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
P = T.KV_PAGE


HALF = "fp16 weights"


def bound(out, size, reach, n, D, dtype, vmax=0.0):
    """(bound of the outputs' error, of lse's)."""
    d = (D + 4) * 2.0 ** -24 * reach + 2 * 2.0 ** -23 * reach
    fp = 2 * d + (n + 40) * 2.0 ** -23
    half = 2.0 ** -24 if dtype == F32 else 2.0 ** -8
    weights = {BF: 2.0 ** -8, HALF: 2.0 ** -11, F32: 0.0}[dtype]
    tol = half * np.abs(out) + (weights + fp[..., None]) * size * (1 + 2.0 ** -7) + 1e-38
    if dtype == HALF:
        tol = tol + n * 2.0 ** -31 * vmax
    return tol, d + (n + 40) * 2.0 ** -23 + 2.0 ** -22 * reach


def check(got, lse, want, D, dtype, n, vmax=0.0):
    out, ref_lse, size, reach = want
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all()
    tol, ltol = bound(out, size, reach, n, D, dtype, vmax)
    bad = np.argwhere(np.abs(g - out) > tol)
    assert bad.size == 0, (f"{len(bad)} of {g.size} values off, worst "
                           f"{np.max(np.abs(g - out) / tol):.2f} of its bound, first {bad[:4].tolist()}")
    z = lse.double().cpu().numpy()
    some = ~np.isinf(ref_lse)
    assert (z[~some] == -np.inf).all()
    z, ref_lse = z[some], ref_lse[some]
    assert (np.abs(z - ref_lse) <= ltol[some] + 2.0 ** -23 * np.abs(ref_lse)).all()


def rows(g, n, H, D, dtype=BF, scale=1.0):
    return (torch.randn(n, H, D, generator=g) * scale).to(dtype).cuda()


# ------------------------------------------------------------------------- attend_window
WINDOW_CASES = [
    # lens, heads, kv_heads, D, dtype, window, sinks
    ([1], 1, 1, 64, BF, 0, 0),
    ([0, 1, 2, 0], 2, 2, 32, BF, 1, 0),
    ([63, 64, 65], 4, 4, 64, BF, 0, 0),
    ([127, 129, 255, 257, 31], 4, 2, 64, BF, 0, 0),
    ([300, 7, 411], 8, 2, 32, BF, 65, 3),
    ([511, 130], 2, 1, 128, BF, 100, 1),
    ([200, 90], 6, 2, 128, BF, 0, 0),
    ([700], 4, 4, 64, BF, 64, 64),
    ([700], 4, 4, 64, BF, 1, 1),
    ([650, 20], 4, 1, 64, BF, 130, 200),
    ([900], 3, 3, 64, BF, 899, 5),
    ([900], 3, 3, 64, BF, 900, 5),
    ([1200], 16, 1, 64, BF, 333, 70),
    ([1], 1, 1, 32, F32, 0, 0),
    ([31, 32, 33, 0, 100], 4, 4, 32, F32, 0, 0),
    ([129, 257], 4, 2, 64, F32, 0, 0),
    ([300, 150], 2, 1, 128, F32, 50, 2),
    ([500], 8, 2, 64, F32, 128, 33),
    ([400], 3, 3, 32, F32, 1, 40),
]


@pytest.mark.parametrize("lens,H,Hkv,D,dtype,window,sinks", WINDOW_CASES)
def test_attend_window(lens, H, Hkv, D, dtype, window, sinks):
    print(f"attend_window {lens} heads {H}/{Hkv} D {D} {dtype} window {window} sinks {sinks}",
          flush=True)
    g = torch.Generator().manual_seed(sum(lens) * 7 + H + D + window)
    total = sum(lens)
    q, k, v = (rows(g, total, h, D, dtype) for h in (H, Hkv, Hkv))
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens)])[:-1].astype(np.int64)).cuda()
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    lse = torch.full((total, H), 7.0, device="cuda")
    out = T.attend_window(q, k, v, off, length, max(lens), window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    at = 0
    for L in lens:
        sl = slice(at, at + L)
        want = history.window_attention(*(x[sl].double().cpu().numpy() for x in (q, k, v)), window, sinks)
        check(out[sl], lse[sl], want, D, dtype, L)
        at += L


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_window_slices_of_one_projection_and_rows_of_nobody(dtype):
    """q, k and v as slices of one buffer; sequences out of order with gaps between and behind, whose
    rows hold NaN and stay as they were; tokens past max_len are not computed."""
    H, Hkv, D = 4, 2, 64
    g = torch.Generator().manual_seed(3)
    rows_total = 700
    buf = torch.full((rows_total, H + 2 * Hkv + 1, D), float("nan"), dtype=dtype, device="cuda")
    spans = [(400, 131), (5, 200), (230, 64), (690, 0)]
    for a, n in spans:
        buf[a:a + n] = rows(g, n, H + 2 * Hkv + 1, D, dtype)
    q, k, v = buf[:, :H], buf[:, H:H + Hkv], buf[:, H + Hkv:H + 2 * Hkv]
    out = torch.full((rows_total, H, D), 5.0, dtype=dtype, device="cuda")
    lse = torch.full((rows_total, H), 5.0, device="cuda")
    off = torch.tensor([a for a, _ in spans]).cuda()
    length = torch.tensor([n for _, n in spans], dtype=torch.int32).cuda()
    T.attend_window(q, k, v, off, length, 150, window=70, sinks=2, scale=0.2, out=out, lse=lse)
    torch.cuda.synchronize()
    mine = torch.zeros(rows_total, dtype=torch.bool, device="cuda")
    for a, n in spans:
        n = min(n, 150)
        sl = slice(a, a + n)
        want = history.window_attention(*(x[sl].double().cpu().numpy() for x in (q, k, v)), 70, 2, 0.2)
        check(out[sl], lse[sl], want, D, dtype, max(n, 1))
        mine[sl] = True
    assert (out[~mine] == 5.0).all() and (lse[~mine] == 5.0).all()


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 64)])
def test_attend_window_extreme_scores(dtype, D):
    """Scores of thousands, growing and falling along the sequence, as one-hot softmaxes are."""
    L, H = 300, 2
    g = torch.Generator().manual_seed(11)
    q, k, v = (rows(g, L, H, D, dtype) for _ in range(3))
    ramp = torch.linspace(-1, 1, L).view(L, 1, 1).cuda()
    for kk in (k * 50 * (1 + ramp), k * 50 * (1 - ramp), k * 1e-30, k * 0):
        kk = kk.to(dtype)
        lse = torch.empty(L, H, device="cuda")
        out = T.attend_window(q, kk, v, torch.zeros(1, dtype=torch.int64).cuda(),
                              torch.tensor([L], dtype=torch.int32).cuda(), L, lse=lse)
        want = history.window_attention(*(x.double().cpu().numpy() for x in (q, kk, v)))
        check(out, lse, want, D, dtype, L)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("spread,scale", [(0.0, 0.0), (2.0 ** -120, 0.0), (0.0, 1e-44), (1.0, 1e-40)])
def test_attend_window_scores_below_fp32(dtype, spread, scale):
    g = torch.Generator().manual_seed(12)
    q, k = rows(g, 100, 2, 64, dtype, spread), rows(g, 100, 2, 64, dtype, spread)
    v, lse = rows(g, 100, 2, 64, dtype), torch.empty(100, 2, device="cuda")
    out = T.attend_window(q, k, v, torch.zeros(1, dtype=torch.int64).cuda(),
                          torch.tensor([100], dtype=torch.int32).cuda(), 100, 30, 2, scale, lse=lse)
    want = history.window_attention(*(x.double().cpu().numpy() for x in (q, k, v)), 30, 2,
                                    scale if scale else None)
    check(out, lse, want, 64, dtype, 100)


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (70, 2 ** 31 - 1),
                                          (0, 2 ** 31 - 1)])
def test_largest_window_and_sinks_are_none(window, sinks):
    L, D = 500, 64
    g = torch.Generator().manual_seed(13)
    q, k, v = (rows(g, L, 2, D) for _ in range(3))
    off, length = torch.zeros(1, dtype=torch.int64).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
    want = T.attend_window(q, k, v, off, length, L)
    got = T.attend_window(q, k, v, off, length, L, window=window, sinks=sinks)
    assert torch.equal(want, got)
    p = Pair(seqs=1, pages=9, blocks=9, H=2, D=D, seed=1)
    p.grow([L])
    q = rows(g, 40, 2, D)
    o2 = torch.tensor([0, 40]).cuda()
    for flags in (T.MASK_NONE, T.MASK_CAUSAL):
        want = T.kv_attend(p.gpu, 0, q, o2, 40, flags=flags)
        got = T.kv_attend(p.gpu, 0, q, o2, 40, flags=flags, window=window, sinks=sinks)
        # (a window may divide the work otherwise)
        assert float((want.float() - got.float()).abs().max()) <= 2.0 ** -7 * float(want.abs().max())


def test_batches_of_no_rows():
    """Requests whose histories are all empty, and an extension by nothing."""
    none = rows(torch.Generator().manual_seed(13), 0, 2, 64)
    off, n = torch.zeros(3, dtype=torch.int64).cuda(), torch.zeros(3, dtype=torch.int32).cuda()
    assert T.attend_window(none, none, none, off, n, 50).shape == (0, 2, 64)
    c = T.KvCache.create(1, 4, 3, 2, 2, 64)
    T.kv_extend(c, n)
    T.kv_append(c, 0, none, none, off, 50)
    assert T.kv_attend(c, 0, none, torch.zeros(4, dtype=torch.int64).cuda(), 0).shape == (0, 2, 64)
    torch.cuda.synchronize()
    assert c.length.tolist() == [0, 0, 0]


def test_attend_window_does_not_see_the_future():
    """NaN and infinities in later tokens' tiles do not reach the rows of earlier tiles."""
    L, H, D = 600, 2, 64
    g = torch.Generator().manual_seed(12)
    q, k, v = (rows(g, L, H, D) for _ in range(3))
    off, length = torch.zeros(1, dtype=torch.int64).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
    want = T.attend_window(q, k, v, off, length, L)
    k2, v2 = k.clone(), v.clone()
    k2[576:], v2[576:] = float("nan"), float("inf")
    got = T.attend_window(q, k2, v2, off, length, L)
    assert torch.equal(want[:512], got[:512])


# ------------------------------------------------------------------------- the cache's state
def new_cache(seqs, pages, blocks, H, D, layers=1, dirty=True):
    c = T.KvCache.create(layers, pages, seqs, blocks, H, D)
    if dirty:   # what the buffers held before does not matter
        for x in (c.k, c.v):
            x.fill_(113)
        for x in (c.k_scale, c.v_scale, c.k_tail, c.v_tail):
            x.fill_(float("nan"))
    return c


class Pair:
    """A cache on the GPU and the oracle's, driven alike."""

    def __init__(self, seqs, pages, blocks, H, D, layers=1, seed=0):
        self.gpu = new_cache(seqs, pages, blocks, H, D, layers)
        self.ref = history.Cache(seqs, pages, blocks, layers)
        self.g = torch.Generator().manual_seed(seed)
        self.seqs, self.layers, self.H, self.D = seqs, layers, H, D

    def grow(self, count, spread=1.0):
        """extend + append of random tokens."""
        off = np.concatenate([[0], np.cumsum(np.maximum(count, 0))])
        total = int(off[-1])
        kv = rows(self.g, max(total, 1) * self.layers, 2 * self.H, self.D, scale=spread)
        kv = kv.view(self.layers, max(total, 1), 2 * self.H, self.D)
        d_off = torch.from_numpy(off).cuda()
        T.kv_extend(self.gpu, torch.tensor(count, dtype=torch.int32).cuda())
        for layer in range(self.layers):
            T.kv_append(self.gpu, layer, kv[layer, :, :self.H], kv[layer, :, self.H:], d_off,
                        max(max(count), 0))
        self.ref.extend(list(count))
        host = kv.double().cpu().numpy()
        self.ref.append(host[:, :, :self.H], host[:, :, self.H:], off)

    def fork(self, parent):
        T.kv_fork(self.gpu, torch.tensor(parent, dtype=torch.int32).cuda())
        self.ref.fork(parent)

    def free(self, drop):
        T.kv_free(self.gpu, torch.tensor(drop, dtype=torch.uint8).cuda())
        self.ref.free(drop)

    def trim(self, window, sinks):
        T.kv_trim(self.gpu, window, sinks)
        self.ref.trim(window, sinks)

    def compact(self):
        used = T.kv_compact(self.gpu)
        assert int(used) == self.ref.compact()

    def vmax(self, s, layer):
        return max((float(np.abs(t[layer]).max()) for t in self.ref.v[s]), default=0.0)

    def same(self, content=True):
        """The whole state: tables, lengths, counts, and what pages and tails hold, exactly."""
        c, r = self.gpu, self.ref
        torch.cuda.synchronize()
        assert c.length.tolist() == r.len
        assert c.fresh.tolist() == r.fresh
        assert c.refs.tolist() == r.refs
        table = c.table.cpu().numpy()
        for s in range(self.seqs):
            want = [-1 if p is None else p for p in r.table[s]]
            assert table[s].tolist() == want + [-1] * (table.shape[1] - len(want)), s
        if not content:
            return
        for s in range(self.seqs):
            for layer in range(self.layers):
                for b, page in enumerate(r.table[s]):
                    if page is None:
                        continue
                    for rows_, codes, scale, turn in ((r.k[s], c.k, c.k_scale, False),
                                                      (r.v[s], c.v, c.v_scale, True)):
                        x = np.stack([t[layer] for t in rows_[b * P:(b + 1) * P]])   # [64, H, D]
                        got = codes[layer, page].cpu().numpy()
                        sc = scale[layer, page].cpu().numpy()
                        for h in range(self.H):
                            q, unit = history.quantise(x[:, h])
                            assert np.array_equal(got[h].T if turn else got[h], q), (s, b, h, turn)
                            assert sc[h] == np.float32(unit)
                n = r.len[s] % P
                if n:
                    kt = c.k_tail[layer, s, :, :n].double().cpu().numpy()
                    vt = c.v_tail[layer, s, :, :, :n].double().cpu().numpy()
                    for h in range(self.H):
                        assert np.array_equal(kt[h], [t[layer][h] for t in r.k[s][-n:]]), (s, h)
                        assert np.array_equal(vt[h].T, [t[layer][h] for t in r.v[s][-n:]]), (s, h)


@pytest.mark.parametrize("D,H", [(32, 3), (64, 2), (128, 1)])
def test_append_in_steps(D, H):
    """Tokens one by one, in chunks that end inside, at and past a block's end, and many blocks at
    once; nothing for some sequences."""
    p = Pair(seqs=5, pages=40, blocks=8, H=H, D=D, layers=2, seed=D)
    for count in ([1, 63, 64, 65, 0], [1, 1, 0, 62, 200], [62, 64, 128, 1, 1], [0, 0, 0, 0, 0],
                  [0, 0, 3, 0, 55], [1, 127, 61, 129, 0]):
        p.grow(count)
        p.same()


def test_append_values_of_every_size():
    """Blocks that are zero, tiny, huge, and full of exact halves."""
    p = Pair(seqs=1, pages=8, blocks=8, H=1, D=64, seed=1)
    for spread in (0.0, 2.0 ** -104, 2.0 ** -99, 1e-20, 3.0, 1e30, 2.0 ** 120):
        p.grow([64], spread)
    p.same()
    q = Pair(seqs=1, pages=2, blocks=2, H=1, D=32, seed=2)
    T.kv_extend(q.gpu, torch.tensor([128], dtype=torch.int32).cuda())
    g = np.random.default_rng(3)
    x = torch.from_numpy(g.integers(-254, 255, size=(128, 2, 32))).to(BF)
    x[0], x[70] = 254, -254
    x[64:] *= 2.0 ** -60
    x = x.cuda()
    T.kv_append(q.gpu, 0, x[:, :1], x[:, 1:], torch.zeros(1, dtype=torch.int64).cuda(), 128)
    q.ref.extend([128])
    h = x.double().cpu().numpy()[None]
    q.ref.append(h[:, :, :1], h[:, :, 1:], [0])
    q.same()


def test_extend_refusals():
    """A sequence past its table is not extended; where the pool runs dry, none from there on is,
    and no page is lost."""
    p = Pair(seqs=6, pages=5, blocks=3, H=1, D=32, seed=4)
    p.grow([70, 256, 10, 64, 0, -5])       # the second would need 4 blocks
    p.same()
    p.grow([60, 64, 70, 130, 1, 0])        # 2 + 1 of 5 pages left for 1 + 1 + ...: the fourth is dry
    p.same()
    p.free([1, 0, 0, 0, 0, 0])
    p.grow([0, 0, 0, 64, 64, 255])
    p.same()
    T.kv_extend(p.gpu, torch.tensor([2 ** 31 - 1] * 6, dtype=torch.int32).cuda())
    p.ref.extend([2 ** 31 - 1] * 6)
    p.same(content=False)


def test_extend_many_sequences_and_pages():
    """More sequences than threads, more pages than one step of the scan, holes everywhere."""
    n, pages = 2500, 9000
    c = new_cache(n, pages, 8, 1, 32, dirty=False)
    ref = history.Cache(n, pages, 8)
    g = np.random.default_rng(6)
    held = g.random(pages) < 0.4
    c.refs.copy_(torch.from_numpy(held.astype(np.int32)))
    ref.refs = [int(x) for x in held]
    for step in range(4):
        count = g.integers(-20, 200, size=n) * (g.random(n) < 0.7)
        T.kv_extend(c, torch.from_numpy(count.astype(np.int32)).cuda())
        ref.extend([int(x) for x in count])
        assert c.fresh.tolist() == ref.fresh, step
        assert c.refs.tolist() == ref.refs and c.length.tolist() == ref.len
    table = c.table.cpu().numpy()
    for s in range(n):
        assert table[s, :len(ref.table[s])].tolist() == ref.table[s]


def test_extend_gives_back_thousands_of_pages():
    """A sequence that the pool proves too small for after most of its pages were found; the sequences
    behind it, which would fit, get none either."""
    c, ref = new_cache(4, 6000, 8000, 1, 32, dirty=False), history.Cache(4, 6000, 8000)
    for count in ([64 * 100, 64 * 7000, 64, 5], [3, 64 * 5900 - 3, 1, 64], [0, 64 * 5901, 64, 0]):
        T.kv_extend(c, torch.tensor(count, dtype=torch.int32).cuda())
        ref.extend(count)
        assert c.fresh.tolist() == ref.fresh and c.length.tolist() == ref.len
        assert c.refs.tolist() == ref.refs
        for s in range(4):
            row = [x for x in c.table[s].tolist() if x != -1]
            assert row == ref.table[s][:len(row)] and len(row) == ref.len[s] // P


def test_the_most_sequences():
    n = T.KV_SEQS_MAX
    c = new_cache(n, 50000, 4, 1, 32, dirty=False)
    ref = history.Cache(n, 50000, 4)
    g = np.random.default_rng(8)
    for step in range(2):
        count = g.integers(0, 140, size=n)
        T.kv_extend(c, torch.from_numpy(count.astype(np.int32)).cuda())
        ref.extend([int(x) for x in count])
        assert c.fresh.tolist() == ref.fresh and c.refs.tolist() == ref.refs
    table = c.table.cpu().numpy()
    assert all(table[s, :len(ref.table[s])].tolist() == ref.table[s] for s in range(n))
    T.kv_trim(c, 2 ** 31 - 1, 2 ** 31 - 1)      # nothing to release, at the largest arguments
    T.kv_free(c, torch.ones(n, dtype=torch.uint8, device="cuda"))
    assert int(c.refs.abs().sum()) == 0 and int((c.table != -1).sum()) == 0


def test_fork_shares_pages_and_copies_tails():
    p = Pair(seqs=8, pages=30, blocks=6, H=2, D=64, layers=2, seed=7)
    p.grow([130, 64, 5, 0, 0, 0, 0, 0])
    #          itself a child; not empty; no such sequence; an empty parent
    p.fork([-1, -1, 0, 0, 0, 3, 99, 7])
    p.same()
    p.fork([-1, -1, -1, -1, -1, 2, 1, -1])
    p.same()
    p.grow([1, 1, 60, 62, 0, 59, 130, 64])     # the copies go their own ways
    p.same()
    p.free([1, 0, 0, 0, 0, 1, 0, 0])
    p.same()
    p.free([0, 1, 1, 1, 1, 0, 1, 1])
    p.same()
    assert int(p.gpu.refs.abs().sum()) == 0 and int((p.gpu.table != -1).sum()) == 0


def test_trim_and_compact():
    p = Pair(seqs=4, pages=64, blocks=16, H=1, D=32, layers=3, seed=8)
    p.grow([1000, 64, 63, 640])
    p.fork([-1, -1, -1, -1])
    p.trim(2000, 0)
    p.same()
    p.trim(10, 2 ** 31 - 1)
    p.same()
    p.trim(300, 65)
    p.same()
    p.trim(300, 65)       # again: nothing more
    p.same()
    p.compact()
    p.same()
    p.compact()           # again: nothing moves
    p.same()
    p.grow([64, 64, 64, 64])
    p.free([0, 1, 0, 0])
    p.compact()
    p.same()
    p.trim(1, 0)
    p.same()
    p.free([1, 1, 1, 1])
    p.compact()
    p.same()


def test_random_walk():
    """Any order of calls leaves the oracle's state."""
    g = np.random.default_rng(9)
    p = Pair(seqs=7, pages=60, blocks=9, H=1, D=32, layers=1, seed=10)
    for step in range(40):
        what = g.choice(["grow", "grow", "grow", "fork", "free", "trim", "compact"])
        if what == "grow":
            p.grow([int(x) for x in g.integers(0, 150, size=7) * (g.random(7) < 0.6)])
        elif what == "fork":
            p.fork([int(x) for x in np.where(g.random(7) < 0.4, g.integers(0, 7, size=7), -1)])
        elif what == "free":
            p.free([int(x) for x in g.random(7) < 0.25])
        elif what == "trim":
            p.trim(int(g.integers(1, 300)), int(g.integers(0, 100)))
        else:
            p.compact()
        p.same(content=step % 8 == 7)
    p.same()


# ------------------------------------------------------------------------- kv_attend
def attend_pair(p, n, heads, causal, window=0, sinks=0, layer=0, scale=0.0, max_len=None, seed=0,
                spread=1.5):
    """kv_attend of n[s] queries for every sequence against the oracle."""
    g = torch.Generator().manual_seed(seed + 77)
    off = np.concatenate([[0], np.cumsum(n)])
    total = int(off[-1])
    q = rows(g, total, heads + 1, p.D, scale=spread)[:, 1:]      # a slice: rows lie further apart
    out = torch.full((total, heads, p.D), 9.0, dtype=BF, device="cuda")
    lse = torch.full((total, heads), 9.0, device="cuda")
    if max_len is not None:
        p.gpu.max_len = max_len
    T.kv_attend(p.gpu, layer, q, torch.from_numpy(off).cuda(), max(n), out=out, lse=lse,
                flags=T.MASK_CAUSAL if causal else T.MASK_NONE, window=window, sinks=sinks, scale=scale)
    torch.cuda.synchronize()
    for s in range(p.seqs):
        sl = slice(int(off[s]), int(off[s + 1]))
        if n[s] == 0:
            continue
        want = p.ref.attend(s, layer, q[sl].double().cpu().numpy(), causal, window, sinks,
                            scale if scale else None)
        check(out[sl], lse[sl], want, p.D, HALF, max(p.ref.len[s], 1), p.vmax(s, layer))
    return q, out, lse


ATTEND_CASES = [
    # lens, queries, kv_heads, heads, D, causal, window, sinks
    ([1], [1], 1, 1, 64, True, 0, 0),
    ([0], [3], 1, 2, 32, False, 0, 0),
    ([5, 0, 64], [1, 1, 1], 2, 2, 64, True, 0, 0),
    ([63, 64, 65, 128, 200], [1, 2, 3, 0, 4], 2, 4, 64, False, 0, 0),
    ([63, 64, 65, 128, 200], [1, 64, 3, 70, 4], 2, 4, 64, True, 0, 0),
    ([10, 300], [20, 5], 1, 1, 64, True, 0, 0),           # more queries than tokens
    ([700, 130], [40, 7], 2, 8, 32, False, 100, 3),
    ([700, 130], [40, 7], 2, 8, 32, True, 100, 70),
    ([640, 641], [100, 33], 1, 4, 128, True, 129, 0),
    ([500, 90, 64], [65, 3, 2], 2, 2, 128, False, 0, 0),
    ([511], [300], 1, 1, 64, True, 1, 0),
    ([1000], [3], 1, 16, 64, False, 1, 1),
    ([2000, 3], [1, 1], 4, 4, 64, False, 0, 0),           # split over workgroups
    ([2500, 900], [2, 1], 1, 2, 32, True, 1500, 5),
    ([3000], [5], 1, 1, 128, False, 0, 0),
]


@pytest.mark.parametrize("lens,n,Hkv,H,D,causal,window,sinks", ATTEND_CASES)
def test_kv_attend(lens, n, Hkv, H, D, causal, window, sinks):
    print(f"kv_attend {lens} queries {n} heads {H}/{Hkv} D {D} causal {causal} window {window} "
          f"sinks {sinks}", flush=True)
    blocks = max(lens) // P + 1
    p = Pair(seqs=len(lens), pages=sum(x // P for x in lens) + 2, blocks=blocks, H=Hkv, D=D, layers=2,
             seed=sum(lens))
    p.grow(lens)
    attend_pair(p, n, H, causal, window, sinks, layer=1)


def test_kv_attend_does_not_depend_on_the_estimate():
    """max_len divides the work; far too small or large ones give the same attention."""
    p = Pair(seqs=2, pages=40, blocks=32, H=2, D=64, seed=21)
    p.grow([1500, 333])
    for max_len in (0, 1, 300, 1500, 10 ** 6, 2 ** 31 - 1):
        attend_pair(p, [2, 3], 4, False, max_len=max_len)


def test_kv_attend_trimmed_pages_are_not_seen():
    p = Pair(seqs=3, pages=60, blocks=20, H=1, D=64, seed=22)
    p.grow([1000, 300, 64])
    p.trim(200, 10)
    attend_pair(p, [4, 4, 4], 2, False, 200, 10)      # the trimmed window: all of it is there
    attend_pair(p, [4, 4, 4], 2, False, 0, 0)         # the whole: what is gone is not seen
    p.trim(1, 0)
    attend_pair(p, [2, 70, 3], 2, False, 0, 0)        # a sequence with nothing left sees nothing


@pytest.mark.parametrize("D,Hkv,heads,causal,window,sinks", [
    (64, 2, 4, False, 0, 0), (64, 1, 1, True, 0, 0), (32, 1, 2, True, 900, 70),
    (128, 1, 4, False, 1500, 1), (64, 4, 4, True, 3000, 0)])
def test_kv_attend_copies_of_one_sequence(D, Hkv, heads, causal, window, sinks):
    """Forks, whose common pages are read once for several of them: next to each other and apart,
    with other sequences between, of different query counts, grown apart by a few tokens, by a block,
    trimmed, and with parents that are gone."""
    print(f"copies: D {D} heads {heads}/{Hkv} causal {causal} window {window} sinks {sinks}", flush=True)
    p = Pair(seqs=19, pages=400, blocks=60, H=Hkv, D=D, seed=D + heads)
    p.grow([2500, 2496, 1300] + [0] * 16)
    #          3..10 of the first, one of the third among them, 12.. of the second
    p.fork([-1] * 3 + [0, 0, 0, 0, 2, 0, 0, 0, -1, 1, 1, 1, 1, 1, -1, 0])
    g = np.random.default_rng(heads)
    most = max(1, 16 * Hkv // heads // 3)
    for step in range(3):
        n = [0, 1, 0] + [int(x) for x in g.integers(0, most + 1, size=16)]
        n[4], n[5] = most, most
        n = [min(x, p.ref.len[s]) if causal else x for s, x in enumerate(n)]
        attend_pair(p, n, heads, causal, window, sinks, seed=step)
        attend_pair(p, [1] * 19, heads, causal, window, sinks, seed=step + 50)
        if step == 0:      # different open blocks, one that fills, one that is left
            p.grow([0, 3, 0, 1, 0, 5, 60, 2, 1, 1, 70, 0, 4, 64, 1, 1, 1, 0, 0])
        elif step == 1:    # the parents go, the copies keep their pages; other sequences take their places
            p.free([1, 1, 0] + [0] * 8 + [1] + [0] * 4 + [1, 0, 0])
            p.grow([100, 2500, 0] + [0] * 16)
            if window:
                p.trim(window, sinks)
    p.same()


def test_kv_attend_copies_give_the_bits_of_sequences_of_their_own():
    """Reading common pages once changes no result: a fork's attention is its parent's."""
    p = Pair(seqs=9, pages=200, blocks=60, H=2, D=64, seed=77)
    p.grow([3333] + [0] * 8)
    p.fork([-1] + [0] * 8)
    g = torch.Generator().manual_seed(5)
    q1 = rows(g, 2, 4, 64)
    one = torch.tensor([0, 2] + [2] * 8).cuda()
    want = T.kv_attend(p.gpu, 0, q1, one, 2, flags=T.MASK_NONE)
    each = torch.arange(10).cuda() * 2
    got = T.kv_attend(p.gpu, 0, q1.repeat(9, 1, 1), each, 2, flags=T.MASK_NONE)
    err = (got.float().view(9, 2, 4, 64) - want.float()).abs().max()
    # (shares divided otherwise: sums of other halves; a rounding to bf16 apart at most)
    assert float(err) <= float(want.float().abs().max()) * 2.0 ** -7
    assert all(torch.equal(got[:2], got[2 * i:2 * i + 2]) for i in range(9))


@pytest.mark.parametrize("n", [1, 16, 17, 33, 64, 65, 130, 700])
def test_kv_attend_every_tile_size(n):
    """16, 32 and 64 query rows a workgroup, and rows beside the last tile."""
    p = Pair(seqs=3, pages=1200, blocks=400, H=4, D=64, seed=n)
    p.grow([16400, 200, 0])
    attend_pair(p, [n, min(n, 3), 1], 4, False, seed=n)
    attend_pair(p, [min(n, 200), min(n, 50), 2], 8, True, 5000, 100, seed=n + 1)


def test_kv_attend_extreme_scales():
    """Blocks whose scales differ by many powers of two, and zero blocks."""
    p = Pair(seqs=1, pages=10, blocks=10, H=1, D=64, seed=23)
    for spread in (1.0, 0.0, 2.0 ** -60, 30.0, 1e-3, 2.0 ** -99, 0.5):
        p.grow([64], spread)
    p.grow([9])
    attend_pair(p, [3], 1, False)
    attend_pair(p, [3], 1, False, scale=2.0)
    attend_pair(p, [70], 1, True, scale=1e-3)


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("spread,keys,scale", [
    (0.0, 0.0, 0.0), (0.0, 2.0 ** -99, 0.0), (2.0 ** -100, 2.0 ** -50, 0.0), (0.0, 1.0, 1e-30),
    (1.0, 1.0, 1e-40), (2.0 ** -120, 1.0, 1e-44)])
def test_kv_attend_scores_below_fp32(n, spread, keys, scale):
    """Queries of zeros or next to it (padding), keys and scales likewise: products of the factors that fp32
    cannot hold are scores of zero, in blocks that are masked in part too."""
    p = Pair(seqs=2, pages=20, blocks=10, H=1, D=64, seed=43)
    p.grow([64, 130], keys)
    p.grow([9, 64], keys)
    attend_pair(p, [n, n], 1, True, spread=spread, scale=scale)
    attend_pair(p, [n, n], 1, False, 100, 3, spread=spread, scale=scale)


@pytest.mark.parametrize("n", [1, 40])
def test_kv_attend_zero_blocks_beside_large_values_and_many(n):
    """Blocks of zero values weigh as much as others: beside values of 2^45, and 40000 tokens of nothing
    else, of which the later ones score higher (their sums pass the earlier reference by 2^13)."""
    p = Pair(seqs=1, pages=10, blocks=10, H=1, D=64, seed=44)
    for spread in (0.0, 2.0 ** 45, 0.0, 0.0, 0.0):
        p.grow([64], spread)
    attend_pair(p, [n], 1, False, spread=2.0 ** -60)

    L, H, D = 40000, 1, 64
    c = T.KvCache.create(1, L // P, 1, L // P, H, D)
    k = torch.full((L, H, D), 1.171875, dtype=BF, device="cuda")
    k[torch.arange(L) // P % 16 < 4] = 0
    v, off = torch.zeros_like(k), torch.zeros(1, dtype=torch.int64).cuda()
    T.kv_extend(c, torch.tensor([L], dtype=torch.int32).cuda())
    T.kv_append(c, 0, k, v, off, L)
    q, lse = torch.ones(n, H, D, dtype=BF, device="cuda"), torch.empty(n, H, device="cuda")
    out = T.kv_attend(c, 0, q, torch.tensor([0, n]).cuda(), n, lse=lse, flags=T.MASK_NONE)
    low = int((k[:, 0, 0] == 0).sum())
    want = np.log(low + (L - low) * np.exp(8 * 1.171875))
    tol = (L + 40) * 2.0 ** -23 + ((D + 4) * 2.0 ** -24 + 2.0 ** -22) * 9.4 + 2.0 ** -23 * want
    assert (out == 0).all() and np.abs(lse.double().cpu().numpy() - want).max() <= tol


def test_steps_of_a_serving_loop():
    """Histories enter, candidates are scored, new actions arrive one at a time, slates fork and
    continue, the window moves on, pages are handed back: every attention against the oracle."""
    p = Pair(seqs=6, pages=80, blocks=20, H=2, D=64, layers=2, seed=24)
    p.grow([500, 70, 900, 0, 0, 0])
    attend_pair(p, [20, 3, 1, 0, 0, 0], 4, False, seed=1)
    for step in range(4):
        p.grow([1, 1, 1, 0, 0, 0])
        attend_pair(p, [1, 1, 1, 0, 0, 0], 4, True, 256, 4, layer=step % 2, seed=step)
    p.fork([-1, -1, -1, 0, 0, 2])
    p.grow([0, 0, 0, 5, 70, 64])
    attend_pair(p, [0, 0, 0, 5, 70, 64], 4, True, seed=9)
    p.trim(256, 4)
    p.compact()
    attend_pair(p, [7, 7, 7, 7, 7, 7], 4, False, 256, 4, layer=1, seed=10)
    p.free([1, 0, 0, 1, 0, 0])
    p.compact()
    attend_pair(p, [1, 1, 1, 1, 1, 1], 2, False, 256, 4, seed=11)
    p.same()


def test_offsets_past_32_bits():
    """A pool of more than 2^31 codes a side: pages at its end."""
    pages, H, D = 135000, 4, 64
    c = T.KvCache.create(1, pages, 2, 10, H, D)
    assert c.k.numel() > 2 ** 31
    c.refs.fill_(1)
    c.refs[-6:] = 0
    off = torch.tensor([0, 200, 400]).cuda()
    g = torch.Generator().manual_seed(31)
    kv = rows(g, 400, 2 * H, D)
    T.kv_extend(c, torch.tensor([200, 200], dtype=torch.int32).cuda())
    T.kv_append(c, 0, kv[:, :H], kv[:, H:], off, 200)
    assert c.table[:, :3].flatten().tolist() == list(range(pages - 6, pages))
    q = rows(g, 4, H, D)
    lse = torch.empty(4, H, device="cuda")
    qoff = torch.tensor([0, 2, 4]).cuda()
    out = T.kv_attend(c, 0, q, qoff, 2, lse=lse, flags=T.MASK_NONE)
    ref = history.Cache(2, 6, 10)
    ref.extend([200, 200])
    h = kv.double().cpu().numpy()[None]
    ref.append(h[:, :, :H], h[:, :, H:], [0, 200])
    for s in range(2):
        want = ref.attend(s, 0, q[2 * s:2 * s + 2].double().cpu().numpy(), False)
        check(out[2 * s:2 * s + 2], lse[2 * s:2 * s + 2], want, D, HALF, 200,
              float(kv.abs().max()))
    c.refs.zero_()
    c.refs[c.table[c.table >= 0].long()] = 1
    assert int(T.kv_compact(c)) == 6      # from the end to the front
    assert c.table[:, :3].flatten().tolist() == list(range(6))
    out2 = T.kv_attend(c, 0, q, qoff, 2, flags=T.MASK_NONE)
    assert torch.equal(out, out2)


# ------------------------------------------------------------------------- streams, graphs
def test_other_stream_and_repeated_calls_give_the_same_bits():
    p = Pair(seqs=3, pages=60, blocks=32, H=2, D=64, seed=41)
    p.grow([1500, 64, 190])
    g = torch.Generator().manual_seed(42)
    q = rows(g, 9, 4, 64)
    off = torch.tensor([0, 3, 6, 9]).cuda()
    want = T.kv_attend(p.gpu, 0, q, off, 3, flags=T.MASK_NONE)
    wq, wk, wv = (rows(g, 333, h, 64) for h in (4, 2, 2))
    o1, l1 = torch.zeros(1, dtype=torch.int64).cuda(), torch.tensor([333], dtype=torch.int32).cuda()
    wwant = T.attend_window(wq, wk, wv, o1, l1, 333, window=50, sinks=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [T.kv_attend(p.gpu, 0, q, off, 3, flags=T.MASK_NONE, stream=side) for _ in range(3)]
    wgot = T.attend_window(wq, wk, wv, o1, l1, 333, window=50, sinks=1, stream=side)
    side.synchronize()
    assert all(torch.equal(want, x) for x in got) and torch.equal(wwant, wgot)


def test_cache_dropped_while_another_stream_reads_it():
    """Memory of a cache that is given up while a call on another stream is still to run is not
    handed out before that call has ended."""
    c = T.KvCache.create(1, 10000, 4, 16, 2, 64)
    old, size = c.k.data_ptr(), c.k.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(int(1e8))   # some 50 ms
    T.kv_trim(c, 5, stream=side)
    del c
    new = torch.empty(size, dtype=torch.int8, device="cuda")
    assert new.data_ptr() != old
    side.synchronize()


def test_graph_of_a_decode_step():
    """extend + append + attend + trim captured once and replayed: every replay is a step of its own
    on the cache's state, with eager work between."""
    H, D, steps = 2, 64, 70
    p = Pair(seqs=2, pages=30, blocks=12, H=H, D=D, seed=51)
    p.grow([250, 60])
    kv = torch.empty(2, 2 * H, D, dtype=BF, device="cuda")
    q = torch.empty(2, H, D, dtype=BF, device="cuda")
    out = torch.empty(2, H, D, dtype=BF, device="cuda")
    lse = torch.empty(2, H, device="cuda")
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 1, 2]).cuda()
    ws = T.Workspace()

    def step():
        T.kv_extend(p.gpu, one)
        T.kv_append(p.gpu, 0, kv[:, :H], kv[:, H:], off, 1)
        T.kv_attend(p.gpu, 0, q, off, 1, out=out, lse=lse, window=200, sinks=2, ws=ws)
        T.kv_trim(p.gpu, 200, 2)

    g = torch.Generator().manual_seed(52)
    graph = None
    for i in range(steps):
        kv.copy_(rows(g, 2, 2 * H, D))
        q.copy_(rows(g, 2, H, D))
        if i == 1:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        p.ref.extend([1, 1])
        h = kv.double().cpu().numpy()[None]
        p.ref.append(h[:, :, :H], h[:, :, H:], [0, 1])
        if i % 8 == 1 or i > steps - 3:
            torch.cuda.synchronize()
            for s in range(2):
                want = p.ref.attend(s, 0, q[s:s + 1].double().cpu().numpy(), True, 200, 2)
                check(out[s:s + 1], lse[s:s + 1], want, D, HALF, p.ref.len[s], p.vmax(s, 0))
        p.ref.trim(200, 2)
    p.same()


def test_graph_of_a_slate_and_an_encoding():
    """fork + extend + append + attend + free + compact and a windowed encoding captured once: every replay
    gives the bits of the eager calls on a cache like it, with eager work between."""
    H, D = 2, 64

    def fresh():
        p = Pair(seqs=4, pages=40, blocks=12, H=H, D=D, seed=61)
        p.grow([250, 130, 0, 0])
        return p.gpu

    a, b = fresh(), fresh()
    parent = torch.tensor([-1, -1, 0, 1], dtype=torch.int32).cuda()
    count = torch.tensor([1, 0, 70, 5], dtype=torch.int32).cuda()
    drop = torch.tensor([0, 0, 1, 1], dtype=torch.uint8).cuda()
    kv = torch.empty(76, 2 * H, D, dtype=BF, device="cuda")
    q = torch.empty(76, H, D, dtype=BF, device="cuda")
    k_off, q_off = torch.tensor([0, 1, 1, 71]).cuda(), torch.tensor([0, 1, 1, 71, 76]).cuda()
    w_off, w_len = torch.tensor([0, 50]).cuda(), torch.tensor([50, 26], dtype=torch.int32).cuda()

    def outputs():
        return [torch.empty(76, H, D, dtype=BF, device="cuda") for _ in range(2)] + [
            torch.empty(1, dtype=torch.int32, device="cuda")]

    def step(c, out, ws):
        T.kv_fork(c, parent)
        T.kv_extend(c, count)
        T.kv_append(c, 0, kv[:, :H], kv[:, H:], k_off, 70)
        T.kv_attend(c, 0, q, q_off, 70, out=out[0], ws=ws[0])
        T.attend_window(q, kv[:, :H], kv[:, H:], w_off, w_len, 50, 20, 1, out=out[1])
        T.kv_free(c, drop)
        T.kv_compact(c, used=out[2], ws=ws[1])

    g = torch.Generator().manual_seed(62)
    ga, gb = outputs(), outputs()
    wa, wb = [T.Workspace(), T.Workspace()], [T.Workspace(), T.Workspace()]
    kv.copy_(rows(g, 76, 2 * H, D))
    q.copy_(rows(g, 76, H, D))
    for c, o, w in ((a, ga, wa), (b, gb, wb)):   # (workspaces and kernels' attributes, outside the capture)
        step(c, o, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, ga, wa)
    for i in range(5):
        kv.copy_(rows(g, 76, 2 * H, D))
        q.copy_(rows(g, 76, H, D))
        graph.replay()
        torch.cuda.synchronize()
        step(b, gb, wb)
        assert all(torch.equal(x, y) for x, y in zip(ga, gb)), i
        assert a.table.tolist() == b.table.tolist() and a.refs.tolist() == b.refs.tolist()
        assert a.length.tolist() == b.length.tolist() == [252 + i, 130, 0, 0]


def test_two_calls_at_once():
    """Calls that only read the cache, on two streams with workspaces of their own."""
    p = Pair(seqs=3, pages=200, blocks=64, H=2, D=64, seed=63)
    p.grow([3500, 640, 2000])
    g = torch.Generator().manual_seed(64)
    qs = [rows(g, 3, 4, 64), rows(g, 3 * 90, 4, 64)]
    offs = [torch.tensor([0, 1, 2, 3]).cuda(), torch.tensor([0, 90, 180, 270]).cuda()]
    want = [T.kv_attend(p.gpu, 0, q, o, n, flags=T.MASK_NONE) for q, o, n in zip(qs, offs, (1, 90))]
    streams, ws = [torch.cuda.Stream() for _ in qs], [T.Workspace() for _ in qs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = [[torch.empty_like(w) for _ in range(4)] for w in want]
    for i in range(4):
        for j in range(2):
            T.kv_attend(p.gpu, 0, qs[j], offs[j], (1, 90)[j], out=outs[j][i], flags=T.MASK_NONE,
                        ws=ws[j], stream=streams[j])
    torch.cuda.synchronize()
    for j in range(2):
        assert all(torch.equal(want[j], x) for x in outs[j])


# ------------------------------------------------------------------------- blocks of very different values
def levels_cache(blocks, seed, copies):
    """A sequence of blocks (tokens, score in nats, spread of the values) for queries of ones, and copies of it:
    the blocks before the last fill pages, all keys of a block are alike."""
    S = 1 + copies
    p = Pair(seqs=S, pages=len(blocks), blocks=len(blocks), H=1, D=64, seed=seed)
    off = torch.zeros(S, dtype=torch.int64).cuda()
    for tokens, score, spread in blocks:
        kv = torch.cat([torch.full((tokens, 1, 64), score / 8.0),
                        torch.randn(tokens, 1, 64, generator=p.g) * spread], 1).to(BF)
        x, count = kv.cuda(), [tokens] + [0] * copies
        T.kv_extend(p.gpu, torch.tensor(count, dtype=torch.int32).cuda())
        T.kv_append(p.gpu, 0, x[:, :1], x[:, 1:], off, tokens)
        p.ref.extend(count)
        h = kv.double().numpy()[None]
        p.ref.append(h[:, :, :1], h[:, :, 1:], [0] * S)
    p.fork([-1] + [0] * copies)
    return p


BIG, SMALL = 2.0 ** 77, 2.0 ** -80


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("blocks", [
    [(64, 0.0, 0.0), (64, 0.0, BIG), (20, 0.0, 1.0)],
    [(64, 0.0, BIG), (64, 3.0, 0.0), (20, 0.0, 1.0)],
    [(64, -3.0, 0.0), (64, 0.0, 2.0 ** 45), (20, 0.0, 1.0)],
    [(64, 0.0, 2.0 ** 45), (64, -3.0, 0.0), (20, 0.0, 1.0)],
    [(64, 0.0, SMALL), (64, 0.0, BIG), (20, 0.0, SMALL)],
    [(64, 0.0, BIG), (64, 2.0, SMALL), (20, 1.0, SMALL)],
    [(64, -10.0, SMALL), (64, -6.0, 0.0), (64, -3.0, 1.0), (64, 0.0, BIG), (20, -3.0, 0.0)],
    [(64, 0.0, BIG), (64, 3.0, 1.0), (64, 6.0, 0.0), (64, 10.0, SMALL), (20, 6.0, 0.0)],
    [(64, 0.0, 2.0 ** 35), (20, 0.0, 0.0)],
    [(64, 0.0, BIG), (20, -5.0, 0.0)],
    [(64, 0.0, 0.0), (64, -4.0, SMALL), (20, 0.0, BIG)],
    [(64, 0.0, 0.0), (20, 1.0, 0.0)],
    [(64, 100.0, SMALL), (64, 0.0, BIG), (20, 50.0, 1.0)],
])
def test_kv_attend_weighs_blocks_whatever_their_values(blocks, n):
    """Zero, tiny and huge values beside each other, in pages and in the open block, in either order and at
    different scores: each token has the weight of its score.  Every block four times over, so that
    a wave meets them one after the other; in one share, and split."""
    print(f"{blocks} n {n}", flush=True)
    copies = 2 if n == 1 else 0   # (rows few enough for copies to share a tile)
    p = levels_cache([b for b in blocks[:-1] for _ in range(4)] + blocks[-1:], n, copies)
    total = n * (1 + copies)
    q, off = torch.ones(total, 1, 64, dtype=BF, device="cuda"), torch.arange(2 + copies).cuda() * n
    want = p.ref.attend(0, 0, np.ones((n, 1, 64)), False)
    for max_len in (0, 64 * 20):
        p.gpu.max_len = max_len
        lse = torch.empty(total, 1, device="cuda")
        out = T.kv_attend(p.gpu, 0, q, off, n, flags=T.MASK_NONE, lse=lse)
        for s in range(0, total, n):
            check(out[s:s + n], lse[s:s + n], want, 64, HALF, p.ref.len[0], p.vmax(0, 0))


# ------------------------------------------------------------------------- what a row's bits depend on
@pytest.mark.parametrize("lens,H,D,dtype,window", [
    ([300], 2, 64, BF, 0), ([300], 2, 128, BF, 100), ([300], 4, 32, BF, 0), ([200], 2, 64, F32, 0),
    ([130, 64, 200] * 70, 4, 64, BF, 0), ([70] * 400, 2, 128, BF, 0)])
def test_attend_window_rows_do_not_depend_on_their_neighbours(lens, H, D, dtype, window):
    """Other rows' queries, whose larger scores move their own references, leave a row's bits alone."""
    g = torch.Generator().manual_seed(71)
    total = sum(lens)
    q, k, v = (rows(g, total, H, D, dtype) for _ in range(3))
    k = (k.float() * torch.linspace(0.2, 3.0, total).view(-1, 1, 1).cuda()).to(dtype)
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens)])[:-1].astype(np.int64)).cuda()
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    mine = torch.arange(total).cuda() % 3 == 1
    got = []
    for others in (1.0, 40.0):
        qq = torch.where(mine[:, None, None], q, (q.float() * others).to(dtype))
        lse = torch.empty(total, H, device="cuda")
        got.append((T.attend_window(qq, k, v, off, length, max(lens), window=window, lse=lse), lse))
    (a, la), (b, lb) = got
    assert torch.equal(a[mine], b[mine]) and torch.equal(la[mine], lb[mine])


@pytest.mark.parametrize("n,D", [(10, 64), (10, 128), (40, 32), (40, 64), (40, 128), (700, 64)])
def test_kv_attend_rows_do_not_depend_on_their_neighbours(n, D):
    g = torch.Generator().manual_seed(72)
    p = Pair(seqs=1, pages=300, blocks=300, H=1, D=D, seed=73)
    for spread in (0.2, 0.6, 1.0, 1.5, 2.0):   # later tokens score higher
        p.grow([1000], spread)
    p.grow([3])
    q = rows(g, n, 1, D)
    mine = torch.arange(n).cuda() % 3 == 1
    got = []
    for others in (1.0, 40.0):
        qq = torch.where(mine[:, None, None], q, (q.float() * others).to(BF))
        for max_len in (0, 5003):
            p.gpu.max_len = max_len
            lse = torch.empty(n, 1, device="cuda")
            got.append((T.kv_attend(p.gpu, 0, qq, torch.tensor([0, n]).cuda(), n, lse=lse,
                                    flags=T.MASK_NONE), lse))
    for (a, la), (b, lb) in zip(got[:2], got[2:]):
        assert torch.equal(a[mine], b[mine]) and torch.equal(la[mine], lb[mine])


@pytest.mark.parametrize("n,heads", [(1, 1), (5, 2), (20, 1), (70, 1), (200, 2)])
def test_kv_attend_weights_round_alike_however_the_work_is_divided(n, heads):
    """A weight is rounded to fp16 against a power of two, so that estimates of the length, by which the pages
    are divided and the references begin, leave its rounding alone.  Scores here are whole eighths of a
    power of two and codes are small, so that the weights are known: fp16 of 2^(j/8), their sum not
    rounded.  fp32's sums of 1000 terms move that quotient by at most 2^-17 of the values' size, and rounding
    to bf16 keeps the order of numbers: an output lies between the roundings of the quotient's bounds."""
    D, L = 64, 1000
    g = np.random.default_rng(n)
    k, v = np.zeros((L, 1, D)), g.integers(-3, 4, size=(L, 1, D)).astype(float)
    j = g.integers(0, 40, size=L)
    k[:, 0, 0], k[::P, 0, 1], v[::P, 0, D - 1] = j / 4.0, 127 / 4.0, 127.0    # key scale 1/4, value scale 1
    c = new_cache(1, L // P, L // P, 1, D)
    off = torch.zeros(1, dtype=torch.int64).cuda()
    kv = torch.from_numpy(np.concatenate([k, v], 1)).to(BF).cuda()
    T.kv_extend(c, torch.tensor([L], dtype=torch.int32).cuda())
    T.kv_append(c, 0, kv[:, :1], kv[:, 1:], off, L)
    q = torch.zeros(n, heads, D, dtype=BF, device="cuda")
    q[:, :, 0] = torch.tensor([1.0, 0.5]).cuda()[torch.arange(n).cuda() % 2][:, None]
    for max_len in (0, 300, 520, 1000, 10 ** 6):
        c.max_len = max_len
        out = T.kv_attend(c, 0, q, torch.tensor([0, n]).cuda(), n, flags=T.MASK_NONE, scale=float(np.log(2.0)))
        for half in range(min(n, 2)):
            w = 2.0 ** ((j / 8.0) if half else (j / 4.0))
            mant, e = np.frexp(w)
            hw = np.ldexp(mant.astype(np.float16).astype(float), e)
            want = hw @ v[:, 0] / w.sum()
            size = hw @ np.abs(v[:, 0]) / w.sum()
            lo, hi = (torch.from_numpy(x).to(BF).double().numpy() for x in (want - 2.0 ** -17 * size,
                                                                            want + 2.0 ** -17 * size))
            got = out[half::2].double().cpu().numpy()
            bad = (got < lo) | (got > hi)
            assert not bad.any(), (max_len, half, int(bad.sum()), got.size)


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_kv_attend_small_weights_in_the_open_block(D, n):
    """63 open tokens of weight 2^-22 beside one token of weight 1 in a page that its wave takes before:
    in the features that the page lacks they are the whole output."""
    p = Pair(seqs=1, pages=4, blocks=4, H=1, D=D, seed=5)
    L = 4 * P + 63
    kv = torch.zeros(L, 2, D)
    unit = D ** -0.5   # a key of x unit scores x against ones
    kv[:4 * P, 0], kv[0, 0], kv[4 * P:, 0] = -40 * unit, 0.0, -15.5 * unit
    kv[0, 1, 0], kv[4 * P:, 1, 1:] = 1.0, 1.0
    kv = kv.to(BF)
    T.kv_extend(p.gpu, torch.tensor([L], dtype=torch.int32).cuda())
    x = kv.cuda()
    T.kv_append(p.gpu, 0, x[:, :1], x[:, 1:], torch.zeros(1, dtype=torch.int64).cuda(), L)
    p.ref.extend([L])
    h = kv.double().numpy()[None]
    p.ref.append(h[:, :, :1], h[:, :, 1:], [0])
    p.gpu.max_len = 0
    lse = torch.empty(n, 1, device="cuda")
    out = T.kv_attend(p.gpu, 0, torch.ones(n, 1, D, dtype=BF, device="cuda"), torch.tensor([0, n]).cuda(),
                      n, flags=T.MASK_NONE, lse=lse)
    check(out, lse, p.ref.attend(0, 0, np.ones((n, 1, D)), False), D, HALF, L, 1.0)


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("scale,queries,keys", [
    (2.0 ** -90, 2.0 ** -33, 2.0 ** 120), (2.0 ** -120, 1.0, 2.0 ** 117), (2.0 ** 90, 2.0 ** -100, 2.0 ** 6),
    (2.0 ** 120, 2.0 ** -30, 2.0 ** -93), (2.0 ** -126, 2.0 ** 100, 2.0 ** 24)])
def test_kv_attend_scores_of_factors_that_lie_far_apart(n, scale, queries, keys):
    """Scores of ordinary size, whatever the sizes of scale, queries and keys that they come from."""
    p = Pair(seqs=1, pages=10, blocks=10, H=1, D=64, seed=47)
    kv = torch.randn(333, 2, 64, generator=p.g)
    kv[:, 0] *= keys
    kv = kv.to(BF)
    x = kv.cuda()
    T.kv_extend(p.gpu, torch.tensor([333], dtype=torch.int32).cuda())
    T.kv_append(p.gpu, 0, x[:, :1], x[:, 1:], torch.zeros(1, dtype=torch.int64).cuda(), 333)
    p.ref.extend([333])
    h = kv.double().numpy()[None]
    p.ref.append(h[:, :, :1], h[:, :, 1:], [0])
    attend_pair(p, [n], 1, True, scale=scale, spread=queries)


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("query,key,scale", [
    ([2.0 ** 100] + [0.0] * 63, [0.0, 2.0 ** 60] + [0.0] * 62, 1e30),     # at right angles
    ([2.0 ** -33] * 64, [2.0 ** 126] * 64, 2.0 ** -100)])                # scores of 1/2
def test_kv_attend_factors_that_fp32_cannot_hold(query, key, scale, n):
    """The scale and the query's size alone leave fp32's range, above or below; with the keys scores are
    ordinary."""
    p = Pair(seqs=1, pages=4, blocks=4, H=1, D=64, seed=48)
    kv = torch.randn(100, 2, 64, generator=p.g)
    kv[:, 0] = torch.tensor(key)
    kv = kv.to(BF)
    x = kv.cuda()
    T.kv_extend(p.gpu, torch.tensor([100], dtype=torch.int32).cuda())
    T.kv_append(p.gpu, 0, x[:, :1], x[:, 1:], torch.zeros(1, dtype=torch.int64).cuda(), 100)
    p.ref.extend([100])
    h = kv.double().numpy()[None]
    p.ref.append(h[:, :, :1], h[:, :, 1:], [0])
    q = torch.tensor(query).to(BF).repeat(n, 1, 1)
    lse = torch.empty(n, 1, device="cuda")
    out = T.kv_attend(p.gpu, 0, q.cuda(), torch.tensor([0, n]).cuda(), n, flags=T.MASK_NONE, scale=scale, lse=lse)
    check(out, lse, p.ref.attend(0, 0, q.double().numpy(), False, scale=scale), 64, HALF, 100, p.vmax(0, 0))


@pytest.mark.parametrize("n", [1, 3, 20, 70])
def test_kv_attend_leaves_the_rows_of_no_sequence(n):
    """A padded batch: rows before the first sequence's and behind the last one's stay as they were, with
    the pages split over workgroups and not."""
    p = Pair(seqs=3, pages=60, blocks=60, H=1, D=64, seed=49)
    p.grow([1500, 64, 130])
    g = torch.Generator().manual_seed(50)
    for before, behind in ((0, 5), (2, 9)):
        counts = [n, 0, n]
        off = np.concatenate([[0], np.cumsum(counts)]) + before
        total = int(off[-1]) + behind
        q = rows(g, total, 2, 64)
        for max_len in (0, 2000):
            p.gpu.max_len = max_len
            out = torch.full((total, 2, 64), 9.0, dtype=BF, device="cuda")
            lse = torch.full((total, 2), 9.0, device="cuda")
            ws = T.Workspace()
            ws.get(1 << 20)
            ws.buf.fill_(255)      # (NaN)
            T.kv_attend(p.gpu, 0, q, torch.from_numpy(off).cuda(), n, out=out, lse=lse,
                        flags=T.MASK_NONE, ws=ws)
            for s in (0, 2):
                sl = slice(int(off[s]), int(off[s + 1]))
                want = p.ref.attend(s, 0, q[sl].double().cpu().numpy(), False)
                check(out[sl], lse[sl], want, 64, HALF, 1500, p.vmax(s, 0))
            for x in (out, lse):
                assert (x[:before] == 9.0).all() and (x[int(off[-1]):] == 9.0).all()


def test_workspace_that_grows_after_a_capture():
    """A captured call's workspace stays its own when a larger call takes the same Workspace afterwards."""
    p = Pair(seqs=1, pages=40, blocks=40, H=1, D=64, seed=51)
    p.grow([2000])
    g = torch.Generator().manual_seed(52)
    q, big = rows(g, 1, 2, 64), rows(g, 90, 2, 64)
    off, off_big = torch.tensor([0, 1]).cuda(), torch.tensor([0, 90]).cuda()
    want = T.kv_attend(p.gpu, 0, q, off, 1, flags=T.MASK_NONE)
    ws, out = T.Workspace(), torch.empty_like(q)
    T.kv_attend(p.gpu, 0, q, off, 1, out=out, flags=T.MASK_NONE, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.kv_attend(p.gpu, 0, q, off, 1, out=out, flags=T.MASK_NONE, ws=ws)
    small = ws.buf.numel()
    T.kv_attend(p.gpu, 0, big, off_big, 90, flags=T.MASK_NONE, ws=ws)
    assert ws.buf.numel() > small
    other = [torch.full((small,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all((x == 77).all() for x in other)


# ------------------------------------------------------------------------- kernels that large batches take
# (tokens of the longer sequences, heads, kv_heads, D, window, sinks); 200 sequences, so that there are more
# workgroups than the kernel with eight waves takes (768)
@pytest.mark.parametrize("long,H,Hkv,D,window,sinks", [
    ([700, 1000], 4, 4, 32, 0, 0), ([700, 1000], 8, 4, 32, 100, 3), ([700, 1000], 4, 4, 64, 0, 0),
    ([513, 900], 8, 4, 64, 65, 70), ([700, 1000], 4, 4, 128, 0, 0), ([700, 899], 6, 3, 128, 200, 5)])
def test_attend_window_large_batches(long, H, Hkv, D, window, sinks):
    """Many short ragged sequences, empty ones among them, and some of several tiles."""
    print(f"{long} heads {H}/{Hkv} D {D} window {window} sinks {sinks}", flush=True)
    g = np.random.default_rng(D + window)
    lens = [int(x) for x in g.integers(1, 131, size=200)]
    for i in range(0, 200, 37):
        lens[i] = 0
    lens[5], lens[120] = long
    assert len(lens) * Hkv * -(-max(lens) * (H // Hkv) // 128) > 768
    gt = torch.Generator().manual_seed(D)
    total = sum(lens)
    q, k, v = (rows(gt, total, h, D) for h in (H, Hkv, Hkv))
    off = np.concatenate([[0], np.cumsum(lens)])
    lse = torch.full((total, H), 7.0, device="cuda")
    out = T.attend_window(q, k, v, torch.from_numpy(off[:-1].astype(np.int64)).cuda(),
                          torch.tensor(lens, dtype=torch.int32).cuda(), max(lens), window=window, sinks=sinks, lse=lse)
    host = [x.double().cpu().numpy() for x in (q, k, v)]
    for a, L in zip(off, lens):
        sl = slice(int(a), int(a) + L)
        check(out[sl], lse[sl], history.window_attention(*(x[sl] for x in host), window, sinks), D, BF, max(L, 1))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("seqs", [96, 97])
def test_attend_window_either_side_of_the_split(seqs, D):
    """768 workgroups, the most that take eight waves, and the next number: the same bits but for the order in
    which halves are joined."""
    H, L = 8, 100
    g = torch.Generator().manual_seed(seqs)
    q, k, v = (rows(g, seqs * L, H, D) for _ in range(3))
    lse = torch.empty(seqs * L, H, device="cuda")
    out = T.attend_window(q, k, v, torch.arange(seqs).cuda() * L,
                          torch.full((seqs,), L, dtype=torch.int32).cuda(), L, window=40, sinks=2, lse=lse)
    for s in (0, 1, seqs // 2, seqs - 1):
        sl = slice(s * L, s * L + L)
        want = history.window_attention(*(x[sl].double().cpu().numpy() for x in (q, k, v)), 40, 2)
        check(out[sl], lse[sl], want, D, BF, L)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("n", [1, 20, 70])
def test_kv_attend_shares_of_many_pages(n, D):
    """An estimate far too small: shares of hundreds of pages, whose numbers a wave looks up 64 at a time."""
    L = 40003
    p = Pair(seqs=2, pages=L // P, blocks=L // P, H=1, D=D, seed=n)
    g = torch.Generator().manual_seed(n)
    kv = rows(g, L, 2, D)
    T.kv_extend(p.gpu, torch.tensor([L, 0], dtype=torch.int32).cuda())
    T.kv_append(p.gpu, 0, kv[:, :1], kv[:, 1:], torch.zeros(2, dtype=torch.int64).cuda(), L)
    T.kv_fork(p.gpu, torch.tensor([-1, 0], dtype=torch.int32).cuda())
    p.ref.extend([L, 0])
    h = kv.double().cpu().numpy()
    p.ref.k[0], p.ref.v[0] = [h[i:i + 1, :1] for i in range(L)], [h[i:i + 1, 1:] for i in range(L)]
    p.ref.fork([-1, 0])
    q = rows(g, 2 * n, 1, D)
    q[n:] = q[:n]
    want = p.ref.attend(0, 0, q[:n].double().cpu().numpy(), False, 30000, 9000)
    bits = []
    for max_len in (0, 1, 10 ** 6):
        p.gpu.max_len = max_len
        lse = torch.empty(2 * n, 1, device="cuda")
        out = T.kv_attend(p.gpu, 0, q, torch.tensor([0, n, 2 * n]).cuda(), n, flags=T.MASK_NONE, window=30000,
                          sinks=9000, lse=lse)
        for s in (0, n):
            check(out[s:s + n], lse[s:s + n], want, D, HALF, L, p.vmax(0, 0))
        bits.append(out)
    assert torch.equal(bits[0], bits[1]) and torch.equal(bits[0][:n], bits[0][n:])


@pytest.mark.parametrize("n", [1, 16, 17, 33, 65, 700, 1300])
@pytest.mark.parametrize("D", [32, 128])
def test_kv_attend_every_tile_size_and_width(n, D):
    """As test_kv_attend_every_tile_size, for the other widths, and sizes at which 64 rows a workgroup are
    taken where there are such kernels."""
    p = Pair(seqs=3, pages=1200, blocks=1300, H=2, D=D, seed=n)
    p.grow([16400, 200, 0])
    attend_pair(p, [n, min(n, 3), 1], 2, False, seed=n)
    attend_pair(p, [min(n, 200), min(n, 50), 2], 4, True, 5000, 100, seed=n + 1)


def test_two_graphs_that_share_a_workspace():
    """Two captured calls of different sizes on one Workspace, replayed in turn with eager work between."""
    p = Pair(seqs=2, pages=80, blocks=60, H=2, D=64, seed=53)
    p.grow([3000, 700])
    g = torch.Generator().manual_seed(54)
    qs = [rows(g, 2, 4, 64), rows(g, 80, 4, 64)]
    offs = [torch.tensor([0, 1, 2]).cuda(), torch.tensor([0, 40, 80]).cuda()]
    want = [T.kv_attend(p.gpu, 0, q, o, n, flags=T.MASK_NONE) for q, o, n in zip(qs, offs, (1, 40))]
    outs, ws, graphs = [torch.empty_like(w) for w in want], T.Workspace(), []
    for i in (0, 1):
        T.kv_attend(p.gpu, 0, qs[i], offs[i], (1, 40)[i], out=outs[i], flags=T.MASK_NONE, ws=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            T.kv_attend(p.gpu, 0, qs[i], offs[i], (1, 40)[i], out=outs[i], flags=T.MASK_NONE, ws=ws)
    for step in range(4):
        for i in ((0, 1), (1, 0))[step % 2]:
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i]), (step, i)
        T.kv_trim(p.gpu, 2 ** 31 - 1)


@pytest.mark.parametrize("seqs", [1, 200])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_attend_window_of_one_token_gives_its_value(seqs, D):
    """A weight that is a row's largest is not rounded: a window of 1 gives v itself, to the bit."""
    L, H, Hkv = 70, 8, 4
    g = torch.Generator().manual_seed(D)
    q, k, v = (rows(g, seqs * L, h, D) for h in (H, Hkv, Hkv))
    out = T.attend_window(q, k, v, torch.arange(seqs).cuda() * L,
                          torch.full((seqs,), L, dtype=torch.int32).cuda(), L, window=1)
    assert torch.equal(out, v.repeat_interleave(H // Hkv, 1))
