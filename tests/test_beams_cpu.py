"""A beam search over resident histories without a GPU: the C ABI's structs and refusals (every
argument error is reported before anything is launched), the binding's, and pins of the oracle
(oracle/beams.py) against brute force."""
import ctypes
import decimal
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import beams, history
from paper_2506_02267_amd import tav2 as T
from test_history_cpu import FAKE, fake_kv, fake_queries

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_header(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tav2.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu %zu %d %d %u %u\\n",'
                   'sizeof(tav2_kv_groups), sizeof(tav2_beams), offsetof(tav2_kv_groups, max_own),'
                   'offsetof(tav2_beams, ld), offsetof(tav2_beams, num_requests),'
                   'offsetof(tav2_beams, eos), TAV2_BEAMS_MAX, TAV2_VOCAB_MAX, TAV2_BEAM_RANKED,'
                   'TAV2_BEAM_IN_PLACE);return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert got == [ctypes.sizeof(T.KvGroupsStruct), ctypes.sizeof(T.Beams),
                   T.KvGroupsStruct.max_own.offset, T.Beams.ld.offset, T.Beams.num_requests.offset,
                   T.Beams.eos.offset, T.BEAMS_MAX, T.VOCAB_MAX, T.BEAM_RANKED, T.BEAM_IN_PLACE]


# ------------------------------------------------------------------------- the C ABI
def fake_groups(**kw):
    a = dict(offset=FAKE, prefix=FAKE, num_groups=2, max_members=2, max_own=10, reserved=0)
    return T.KvGroupsStruct(**{**a, **kw})


def fake_beams(**kw):
    a = dict(logits=FAKE, score=FAKE, done=FAKE, allowed=FAKE, ld=1000, allowed_ld=125, num_requests=3,
             beams=4, vocab=1000, dtype=T.BF16, eos=5, reserved=0)
    return T.Beams(**{**a, **kw})


def reorder(c=None, g=None, parent=FAKE, members=4):
    c, g = c or fake_kv(), g or fake_groups()
    return T.load_library().tav2_kv_reorder(ctypes.byref(c), ctypes.byref(g), parent, members, None)


def attend(c=None, g=None, q=None, layer=0, flags=0, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    c, g, q = c or fake_kv(), g or fake_groups(), q or fake_queries()
    return T.load_library().tav2_kv_attend_prefix(ctypes.byref(c), layer, ctypes.byref(g),
                                                  ctypes.byref(q), flags, out, FAKE, ws, ws_bytes, None)


def select(b=None, keep=4, flags=0, parent=FAKE, token=FAKE, score=FAKE, done=FAKE, ws=FAKE,
           ws_bytes=1 << 40):
    b = b or fake_beams()
    return T.load_library().tav2_beam_select(ctypes.byref(b), keep, flags, parent, token, score, done,
                                             ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(num_groups=-1), -2), (dict(max_members=0), -2), (dict(max_members=-3), -2),
    (dict(max_members=T.BEAMS_MAX + 1), -2), (dict(max_own=-1), -2),
    (dict(num_groups=T.KV_SEQS_MAX + 1), -4), (dict(offset=None), -1),
])
def test_groups_are_refused(kw, status):
    assert reorder(g=fake_groups(**kw)) == status
    assert attend(g=fake_groups(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), -1), (dict(len=None), -1), (dict(num_seqs=0), -2), (dict(head_dim=96), -4),
    (dict(v_tail=FAKE + 4), -2)])
def test_caches_are_refused(kw, status):
    assert reorder(c=fake_kv(**kw)) == status
    assert attend(c=fake_kv(**kw)) == status


def test_reorder_argument_errors():
    lib = T.load_library()
    c, g = fake_kv(), fake_groups()
    assert lib.tav2_kv_reorder(None, ctypes.byref(g), FAKE, 4, None) == -1
    assert lib.tav2_kv_reorder(ctypes.byref(c), None, FAKE, 4, None) == -1
    assert reorder(parent=None) == -1
    assert reorder(members=-1) == -2
    assert reorder(members=0, parent=None) == 0
    assert reorder(g=fake_groups(num_groups=0, offset=None, prefix=None)) == 0
    big = fake_kv(num_seqs=T.KV_SEQS_MAX, layers=30000)
    assert reorder(c=big, g=fake_groups(num_groups=T.KV_SEQS_MAX)) == -4


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(offset=None), -1), (dict(total=-1), -2), (dict(max_count=11), -2),
    (dict(max_count=0), -2), (dict(heads=3), -2), (dict(heads=0), -2), (dict(window=-1), -2),
    (dict(sinks=-1), -2), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2), (dict(ld=250), -2),
    (dict(ld=128), -2), (dict(q=FAKE + 8), -2), (dict(heads=131072, ld=1 << 23), -4),
    (dict(total=2 ** 40, max_count=4), -4), (dict(total=2 ** 28, max_count=2 ** 28), -4)])
def test_prefix_queries_are_refused(kw, status):
    assert attend(q=fake_queries(**kw)) == status


def test_prefix_argument_errors():
    lib = T.load_library()
    c, g, q = fake_kv(), fake_groups(), fake_queries()
    b = ctypes.byref
    assert lib.tav2_kv_attend_prefix(b(c), 0, None, b(q), 0, FAKE, None, FAKE, 1 << 40, None) == -1
    assert lib.tav2_kv_attend_prefix(b(c), 0, b(g), None, 0, FAKE, None, FAKE, 1 << 40, None) == -1
    assert attend(g=fake_groups(prefix=None)) == -1
    assert attend(layer=2) == -2 and attend(layer=-1) == -2
    assert attend(flags=2) == -2
    assert attend(out=None) == -1 and attend(out=FAKE + 8) == -2
    need = lib.tav2_kv_attend_prefix_workspace(b(c), b(g), b(q))
    assert need > 0
    assert attend(ws=None) == -5 and attend(ws_bytes=need - 1) == -5 and attend(ws=FAKE + 64) == -5
    assert attend(q=fake_queries(total=0, max_count=0, q=None, offset=None), out=None, ws=None) == 0
    assert attend(g=fake_groups(num_groups=0, offset=None, prefix=None), ws=None) == 0
    assert lib.tav2_kv_attend_prefix_workspace(b(c), b(g), b(fake_queries(heads=3))) == 0
    # the largest sizes: refused, whatever their products
    huge = fake_kv(num_seqs=T.KV_SEQS_MAX, kv_heads=32767, layers=2, max_blocks=1 << 20, max_len=1 << 26)
    assert attend(c=huge, g=fake_groups(num_groups=T.KV_SEQS_MAX, max_members=T.BEAMS_MAX),
                  q=fake_queries(heads=32767, ld=32767 * 64, total=65000, max_count=65000)) == -4


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), -1), (dict(dtype=T.I8), -3), (dict(dtype=7), -3), (dict(num_requests=-1), -2),
    (dict(beams=0), -2), (dict(beams=T.BEAMS_MAX + 1), -2), (dict(vocab=0), -2),
    (dict(vocab=T.VOCAB_MAX + 1, ld=T.VOCAB_MAX + 1, allowed=None), -2), (dict(ld=999), -2),
    (dict(allowed_ld=124), -2), (dict(allowed_ld=-1), -2), (dict(eos=1000), -2),
    (dict(logits=FAKE + 1), -2), (dict(logits=FAKE + 2, dtype=T.F32), -2),
    (dict(beams=1024, vocab=1 << 22, ld=1 << 22, allowed=None), -4),
    (dict(num_requests=1 << 30), -4), (dict(ld=1 << 60), -4), (dict(allowed_ld=1 << 60), -4),
    (dict(num_requests=1 << 24, beams=1, vocab=1 << 20, ld=1 << 20, allowed=None), -4),
])
def test_beams_are_refused(kw, status):
    assert select(fake_beams(**kw)) == status


def test_select_argument_errors():
    lib = T.load_library()
    assert lib.tav2_beam_select(None, 4, 0, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == -1
    assert select(keep=0) == -2 and select(keep=T.K_MAX + 1) == -2
    assert select(flags=2) == -2
    assert select(keep=3, flags=T.BEAM_IN_PLACE) == -2
    assert select(parent=None) == -1 and select(token=None) == -1 and select(score=None) == -1
    need = lib.tav2_beam_select_workspace(ctypes.byref(fake_beams()), 4)
    if need:
        assert select(ws=None) == -5 and select(ws_bytes=need - 1) == -5 and select(ws=FAKE + 4) == -5
    assert lib.tav2_beam_select_workspace(ctypes.byref(fake_beams(beams=0)), 4) == 0
    assert select(fake_beams(num_requests=0, logits=None), parent=None, ws=None) == 0
    large = fake_beams(vocab=100000, ld=100000, allowed=None)
    need = lib.tav2_beam_select_workspace(ctypes.byref(large), 4)
    assert need > 0
    assert select(large, ws=None) == -5 and select(large, ws_bytes=need - 1) == -5
    assert select(large, ws=FAKE + 128) == -5


# ------------------------------------------------------------------------- the binding
def test_binding_refuses():
    z = torch.zeros(6, 10)
    ok = dict(beams=3, keep=2)
    for bad in (z.double(), z.half(), z[0], z.t(), z[:, ::2]):
        with pytest.raises(ValueError):
            T.beam_select(bad, **ok)
    for kw in (dict(beams=4), dict(beams=0), dict(score=torch.zeros(6)), dict(score=torch.zeros(2, 3).double()),
               dict(done=torch.zeros(2, 3)), dict(allowed=torch.zeros(6, 1, dtype=torch.uint8)),
               dict(allowed=torch.zeros(2, 2, dtype=torch.uint8)), dict(allowed=torch.zeros(6, 2)),
               dict(keep=2 ** 33), dict(eos=2 ** 33), dict(eos=-2 ** 40), dict(flags=2 ** 33),
               dict(out=(torch.zeros(2, 2),) * 4)):
        with pytest.raises(ValueError):
            T.beam_select(z, **{**ok, **kw})
    with pytest.raises(ValueError, match="GPU"):
        T.beam_select(z, **ok)


def test_groups_binding_refuses():
    o = torch.zeros(3, dtype=torch.int32)
    for args in ((o.long(),), (o[None],), (o[:0],), (o, torch.zeros(3, dtype=torch.int32)), (o, torch.zeros(2))):
        with pytest.raises(ValueError):
            T.KvGroups(*args)
    with pytest.raises(ValueError):
        T.KvGroups(o, max_members=2 ** 33)
    g = T.KvGroups(o, torch.zeros(2, dtype=torch.int32), max_members=3)
    with pytest.raises(ValueError):
        g.max_own = 2 ** 33
    c = T.KvCache.create(1, 4, 5, 2, 2, 32, device="cpu")
    with pytest.raises(ValueError):
        T.kv_reorder(c, g, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        T.kv_reorder(c, g, torch.zeros(4, dtype=torch.int32))
    q, off = torch.zeros(3, 4, 32, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int64)
    for kw in (dict(q=q.float()), dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), dict(offset=off[:5]),
               dict(offset=off.int()), dict(out=q.float()), dict(lse=torch.zeros(3)), dict(window=2 ** 32),
               dict(layer=2 ** 33), dict(max_count=2 ** 32), dict(scale=1e-60), dict(flags=2 ** 32)):
        a = {**dict(q=q, offset=off, max_count=1), **kw}
        with pytest.raises(ValueError):
            T.kv_attend_prefix(c, a.pop("layer", 0), g, a.pop("q"), a.pop("offset"), a.pop("max_count"), **a)
    with pytest.raises(ValueError, match="GPU"):
        T.kv_attend_prefix(c, 0, g, q, off, 1, ws=T.Workspace("cpu"))


# ------------------------------------------------------------------------- the oracle
def test_select_by_hand():
    """Two beams of three tokens, worth p = 1/2 and 1/4 so far."""
    z = np.log([[0.7, 0.2, 0.1], [0.05, 0.9, 0.05]])
    score = [[math.log(0.5), math.log(0.25)]]
    # 0.35 0.1 0.05 and 0.0125 0.225 0.0125
    p, t, v, e = beams.select(z, 2, 4, score, eos=1)
    assert p.tolist() == [[0, 1, 0, 0]] and t.tolist() == [[0, 1, 1, 2]]
    assert np.allclose(np.exp(v), [[0.35, 0.225, 0.1, 0.05]]) and e.tolist() == [[0, 1, 1, 0]]
    # the first finished: it is one continuation, worth 1/2
    p, t, v, e = beams.select(z, 2, 5, score, done=[[1, 0]], eos=1)
    assert p.tolist() == [[0, 1, 1, 1, -1]] and t.tolist() == [[1, 1, 0, 2, -1]]
    assert np.allclose(np.exp(v), [[0.5, 0.225, 0.0125, 0.0125, 0.0]]) and e.tolist() == [[1, 1, 0, 0, 0]]
    # tokens that are not allowed keep their share of the sum
    p, t, v, e = beams.select(z, 2, 2, score, allowed=np.array([[0, 1, 1], [1, 0, 0]], dtype=bool))
    assert p.tolist() == [[0, 0]] and t.tolist() == [[1, 2]] and np.allclose(np.exp(v), [[0.1, 0.05]])


def test_select_against_all_continuations():
    g = np.random.default_rng(1)
    for _ in range(50):
        R, B, V, K = (int(g.integers(1, n)) for n in (4, 6, 9, 12))
        z = g.integers(-4, 5, size=(R * B, V)) / 2.0      # ties among a beam's tokens
        z[g.random(z.shape) < 0.1] = -np.inf
        z[g.random(z.shape) < 0.05] = np.nan
        score = -g.random((R, B))
        done = g.random((R, B)) < 0.2
        allowed = g.random(z.shape) < 0.8
        p, t, v, e = beams.select(z, B, K, score, done, allowed, eos=0)
        for r in range(R):
            every = []
            for b in range(B):
                if done[r, b]:
                    every.append((-score[r, b], b, 0))
                    continue
                w = [math.exp(x) if math.isfinite(x) else 0.0 for x in z[r * B + b]]
                for i, x in enumerate(w):
                    if x and allowed[r * B + b, i]:
                        every.append((-(score[r, b] + math.log(x / sum(w))), b, i))
            n = min(K, len(every))
            assert np.allclose(v[r, :n], [-c for c, _, _ in sorted(every)[:n]])
            assert len(set(zip(p[r, :n], t[r, :n]))) == n and (p[r, n:] == -1).all()
            value = {(b, i): -c for c, b, i in every}
            assert all(math.isclose(value[(p[r, k], t[r, k])], v[r, k], abs_tol=1e-12) for k in range(n))
            for k in range(n - 1):                # equal ones of a beam: the lower token first
                if p[r, k] == p[r, k + 1] and v[r, k] == v[r, k + 1]:
                    assert t[r, k] < t[r, k + 1]


def by_definition(z, keep, score):
    """(beam, token, score + log(e^z / sum of e^z)) of the `keep` best of one request, in decimals of 120 digits."""
    d = decimal.Decimal
    with decimal.localcontext() as ctx:
        ctx.prec = 120
        every = []
        for b, row in enumerate(np.asarray(z, dtype=np.float64)):
            row = [d(float(x)) for x in row]
            m = max(row)
            total, exps = d(0), {}
            for x in row:
                if x not in exps:
                    exps[x] = (x - m).exp() if x - m > -2000 else d(0)
                total += exps[x]
            base = d(float(score[b])) - total.ln() - m
            every += [(-(base + x), b, v) for v, x in enumerate(row)]
        return [(b, v, float(-c)) for c, b, v in sorted(every)[:keep]]


def large_logits(V, dtype):
    """(logits, scores, keep): rows of logits so large that their own size drowns the logarithm of their sum."""
    g = torch.Generator().manual_seed(V)
    top = torch.finfo(dtype).max
    normal = torch.randn(V, generator=g)
    flat = lambda x: torch.full((V,), x)
    masked = flat(-top)
    masked[V // 3], masked[V - 1] = 0.0, -1.5
    spike = flat(-top)
    spike[V // 2] = top
    steps = flat(2.0 ** 30)
    steps[1::2] = -(2.0 ** 30)
    # a beam whose tokens are all masked by the type's lowest value; all of one size; a few of each
    for rows, score, keep in (([normal, flat(-top)], (0.0, 0.0), 4), ([normal, flat(-top), normal * 3], (-9.0, -0.5, -30.0), 9),
                              ([flat(2.0 ** 30)], (0.0,), 2), ([flat(2.0 ** 24), flat(-top), flat(top), flat(0.0)], (-1.0, -0.25, -0.5, 0.0), 7),
                              ([masked, spike, normal], (-2.0, -1.0, 0.0), 5), ([steps, flat(1.0)], (-0.5, 0.25), 6)):
        z = torch.stack(rows).to(dtype)
        yield z, score, min(keep, z.numel())


@pytest.mark.parametrize("V", [2, 3, 100, 3000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select_of_large_logits(V, dtype):
    for z, score, keep in large_logits(V, dtype):
        p, t, v, _ = beams.select(z.double().numpy(), len(z), keep, [score])
        want = by_definition(z.double().numpy(), keep, score)
        assert list(zip(p[0], t[0])) == [x[:2] for x in want]
        assert np.allclose(v[0], [x[2] for x in want], rtol=2.0 ** -50, atol=2.0 ** -45)


def test_select_in_place():
    """The same beams; those that go on have their best continuation where they are."""
    g = np.random.default_rng(2)
    for _ in range(30):
        R, B, V = (int(g.integers(1, n)) for n in (4, 9, 7))
        z, score = g.normal(size=(R * B, V)), -2 * g.random((R, B))
        score[g.random((R, B)) < 0.2] = -np.inf
        a = beams.select(z, B, B, score)
        b = beams.select(z, B, B, score, in_place=True)
        for r in range(R):
            assert sorted(zip(*(x[r] for x in a))) == sorted(zip(*(x[r] for x in b)))
            for i in range(B):
                mine = a[2][r][a[0][r] == i]
                if len(mine):
                    assert b[0][r, i] == i and b[2][r, i] == mine.max()


def test_reorder_oracle():
    g = np.random.default_rng(3)
    c = history.Cache(7, 60, 8)
    count = [70, 5, 130, 64, 0, 200, 9]
    c.extend(count)
    off = np.concatenate([[0], np.cumsum(count)])
    kv = g.normal(size=(1, off[-1], 1, 4))
    c.append(kv, kv, off)
    was = [(list(t), n, list(k)) for t, n, k in zip(c.table, c.len, c.k)]
    beams.reorder(c, [1, 4, 7], [1, 2, 0, 2, 0, -1])      # a cycle; sequences 4, 5, 6 become 6, 4 and empty
    now = [(t, n, k) for t, n, k in zip(c.table, c.len, c.k)]
    assert now[0] == was[0] and now[1:4] == [was[2], was[3], was[1]]
    assert now[4] == was[6] and now[5] == was[4] and now[6] == ([], 0, [])
    held = [p for t in c.table for p in t]
    assert c.refs == [held.count(p) for p in range(60)]


def test_attend_prefix_oracle():
    """As one sequence of both."""
    g = np.random.default_rng(4)
    c, one = history.Cache(2, 20, 8), history.Cache(1, 20, 16)
    kv = g.normal(size=(2, 1, 192 + 70, 2, 8))
    c.extend([192, 70])
    c.append(kv[0], kv[1], [0, 192])
    one.extend([262])
    one.append(kv[0], kv[1], [0])
    q = g.normal(size=(3, 4, 8))
    for causal in (True, False):
        for window, sinks in ((0, 0), (100, 7), (1, 0), (300, 2)):
            a = beams.attend_prefix(c, 0, 1, 0, q, causal, window, sinks)
            b = one.attend(0, 0, q, causal, window, sinks)
            assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])
    a, b = beams.attend_prefix(c, -1, 1, 0, q, True), c.attend(1, 0, q, True)
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])
