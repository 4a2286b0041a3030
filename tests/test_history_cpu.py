"""Attention over whole histories without a GPU: the C ABI's structs and refusals (every
argument error is reported before anything is launched), the binding's, and pins of the oracle
(oracle/history.py) against brute force."""
import ctypes
import math
import os
import subprocess
import weakref
from fractions import Fraction
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import history
from paper_2506_02267_amd import tav2 as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # an aligned non-null "device" address; never dereferenced on error paths


def test_struct_layouts_match_header(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tav2.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu %d %d\\n",'
                   'sizeof(tav2_window), sizeof(tav2_kv), sizeof(tav2_kv_queries),'
                   'offsetof(tav2_window, scale), offsetof(tav2_window, offset),'
                   'offsetof(tav2_kv, max_len), offsetof(tav2_kv_queries, scale),'
                   'TAV2_KV_PAGE, TAV2_KV_SEQS_MAX);return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert got == [ctypes.sizeof(T.Window), ctypes.sizeof(T.Kv), ctypes.sizeof(T.KvQueries),
                   T.Window.scale.offset, T.Window.offset.offset, T.Kv.max_len.offset,
                   T.KvQueries.scale.offset, T.KV_PAGE, T.KV_SEQS_MAX]


def fake_window(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_ld=256, k_ld=128, v_ld=128, out=FAKE, lse=FAKE, offset=FAKE,
             len=FAKE, num_requests=2, max_len=100, heads=4, kv_heads=2, head_dim=64,
             dtype=T.BF16, window=10, sinks=2, scale=0.0, reserved=0)
    return T.Window(**{**a, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1),
    (dict(offset=None), -1), (dict(len=None), -1),
    (dict(dtype=T.I8), -3), (dict(dtype=9), -3),
    (dict(num_requests=-1), -2), (dict(max_len=-1), -2), (dict(heads=0), -2), (dict(heads=3), -2),
    (dict(kv_heads=0), -2), (dict(window=-1), -2), (dict(sinks=-1), -2), (dict(scale=-1.0), -2),
    (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2),
    (dict(q_ld=255), -2), (dict(q_ld=248), -2), (dict(q_ld=(1 << 24) + 8), -2), (dict(k_ld=120), -2), (dict(v_ld=132), -2),
    (dict(q=FAKE + 8), -2), (dict(k=FAKE + 2), -2), (dict(v=FAKE + 4), -2), (dict(out=FAKE + 8), -2),
    (dict(head_dim=48, q_ld=192, k_ld=96, v_ld=96), -4), (dict(head_dim=256, q_ld=1024), -4),
    (dict(max_len=1 << 30), -4), (dict(num_requests=1 << 30, max_len=1 << 20), -4),
])
def test_attend_window_argument_errors(kw, status):
    a = fake_window(**kw)
    assert T.load_library().tav2_attend_window(ctypes.byref(a), None) == status


def test_attend_window_null_and_empty():
    lib = T.load_library()
    assert lib.tav2_attend_window(None, None) == -1
    for kw in (dict(num_requests=0), dict(max_len=0)):
        a = fake_window(q=None, k=None, v=None, out=None, **kw)
        assert lib.tav2_attend_window(ctypes.byref(a), None) == 0


def fake_kv(**kw):
    a = {n: FAKE for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "table", "len",
                           "fresh", "refs")}
    a.update(num_seqs=4, layers=2, pages=100, max_blocks=16, kv_heads=2, head_dim=64, max_len=900,
             reserved=0)
    return T.Kv(**{**a, **kw})


def fake_queries(**kw):
    a = dict(q=FAKE, offset=FAKE, total=10, ld=256, max_count=4, heads=4, window=0, sinks=0,
             scale=0.0, reserved=0)
    return T.KvQueries(**{**a, **kw})


def kv_calls(c):
    """Every entry point on cache struct c (None: a null pointer), with valid other arguments."""
    lib = T.load_library()
    p = None if c is None else ctypes.byref(c)
    q = ctypes.byref(fake_queries())
    return {"extend": lib.tav2_kv_extend(p, FAKE, None),
            "append": lib.tav2_kv_append(p, 0, FAKE, 128, FAKE, 128, FAKE, 5, None),
            "attend": lib.tav2_kv_attend(p, 0, q, 0, FAKE, FAKE, FAKE, 1 << 40, None),
            "fork": lib.tav2_kv_fork(p, FAKE, None), "free": lib.tav2_kv_free(p, FAKE, None),
            "trim": lib.tav2_kv_trim(p, 10, 2, None),
            "compact": lib.tav2_kv_compact(p, FAKE, FAKE, 1 << 40, None)}


@pytest.mark.parametrize("kw,status", [
    *[({n: None}, -1) for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "table", "len",
                                "fresh", "refs")],
    (dict(num_seqs=0), -2), (dict(layers=0), -2), (dict(pages=0), -2), (dict(max_blocks=0), -2),
    (dict(kv_heads=0), -2), (dict(max_len=-1), -2), (dict(k=FAKE + 8), -2), (dict(v=FAKE + 1), -2),
    (dict(k_tail=FAKE + 2), -2), (dict(v_tail=FAKE + 4), -2),
    (dict(num_seqs=T.KV_SEQS_MAX + 1), -4), (dict(max_blocks=(1 << 20) + 1), -4),
    (dict(head_dim=16), -4), (dict(head_dim=96), -4), (dict(layers=40000, kv_heads=2), -4),
])
def test_every_cache_call_refuses_a_bad_cache(kw, status):
    assert set(kv_calls(fake_kv(**kw)).values()) == {status}
    lib, c = T.load_library(), fake_kv(**kw)
    assert lib.tav2_kv_attend_workspace(ctypes.byref(c), ctypes.byref(fake_queries())) == 0
    assert lib.tav2_kv_compact_workspace(ctypes.byref(c)) == 0


@pytest.mark.parametrize("scale,status", [(2.3e38, 0), (2.37e38, -2), (3.0e38, -2)])
def test_scales_that_log2_e_takes_past_fp32(scale, status):
    """Scores are taken in powers of two: with a scale past FLT_MAX / log2(e) = 2.36e38 a score of zero
    would be 0 times infinity."""
    lib, a, c = T.load_library(), fake_window(num_requests=0, scale=scale), fake_kv()
    assert lib.tav2_attend_window(ctypes.byref(a), None) == status
    q = fake_queries(q=None, offset=None, total=0, max_count=0, scale=scale)
    assert lib.tav2_kv_attend(ctypes.byref(c), 0, ctypes.byref(q), 0, None, None, None, 0, None) == status


def test_null_cache():
    assert set(kv_calls(None).values()) == {-1}


def test_cache_call_argument_errors():
    lib, c = T.load_library(), fake_kv()
    p = ctypes.byref(c)
    assert lib.tav2_kv_extend(p, None, None) == -1
    assert lib.tav2_kv_fork(p, None, None) == -1
    assert lib.tav2_kv_free(p, None, None) == -1
    assert lib.tav2_kv_trim(p, 0, 0, None) == -2
    assert lib.tav2_kv_trim(p, 5, -1, None) == -2
    assert lib.tav2_kv_compact(p, None, FAKE, 1 << 40, None) == -1
    need = lib.tav2_kv_compact_workspace(p)
    assert need > 0
    assert lib.tav2_kv_compact(p, FAKE, None, need, None) == -5
    assert lib.tav2_kv_compact(p, FAKE, FAKE, need - 1, None) == -5
    assert lib.tav2_kv_compact(p, FAKE, FAKE + 64, need, None) == -5

    def append(layer=0, k=FAKE, kl=128, v=FAKE, vl=128, off=FAKE, n=5):
        return lib.tav2_kv_append(p, layer, k, kl, v, vl, off, n, None)

    assert append(layer=2) == append(layer=-1) == append(n=-1) == -2
    assert append(kl=120) == append(vl=130) == append(k=FAKE + 8) == append(v=FAKE + 2) == -2
    assert append(k=None) == append(v=None) == append(off=None) == -1
    assert append(k=None, v=None, off=None, n=0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(offset=None), -1), (dict(total=-1), -2), (dict(max_count=-1), -2),
    (dict(max_count=11), -2), (dict(max_count=0), -2), (dict(heads=0), -2), (dict(heads=3), -2),
    (dict(ld=248), -2), (dict(ld=260), -2), (dict(window=-1), -2), (dict(sinks=-1), -2),
    (dict(scale=-0.5), -2), (dict(scale=float("nan")), -2), (dict(q=FAKE + 8), -2),
    (dict(total=1 << 40, max_count=1), -4), (dict(heads=65536, ld=65536 * 64), -4),
])
def test_attend_query_errors(kw, status):
    lib, c, q = T.load_library(), fake_kv(), fake_queries(**kw)
    st = lib.tav2_kv_attend(ctypes.byref(c), 0, ctypes.byref(q), 0, FAKE, FAKE, FAKE, 1 << 50, None)
    assert st == status


def test_attend_other_errors():
    lib, c, q = T.load_library(), fake_kv(max_len=16384, max_blocks=256), fake_queries()
    p, a = ctypes.byref(c), ctypes.byref(q)
    need = lib.tav2_kv_attend_workspace(p, a)
    assert need > 0 and need % 256 == 0
    call = lambda layer=0, flags=0, out=FAKE, ws=FAKE, n=need, qq=a: lib.tav2_kv_attend(  # noqa: E731
        p, layer, qq, flags, out, None, ws, n, None)
    assert call(layer=2) == call(layer=-1) == call(flags=2) == call(out=FAKE + 8) == -2
    assert call(out=None) == call(qq=None) == -1
    assert call(ws=None) == call(n=need - 1) == call(ws=FAKE + 128) == -5
    empty = fake_queries(q=None, offset=None, total=0, max_count=0)
    assert call(out=None, ws=None, n=0, qq=ctypes.byref(empty)) == 0


def test_sizes_whose_products_pass_64_bits_or_a_launch():
    lib, c = T.load_library(), fake_kv()
    for kw in (dict(total=1 << 62, max_count=1), dict(total=(1 << 63) - 1, max_count=1)):
        q = fake_queries(**kw)
        assert lib.tav2_kv_attend(ctypes.byref(c), 0, ctypes.byref(q), 0, FAKE, FAKE, None, 0,
                                  None) == -4
    wide = fake_kv(num_seqs=T.KV_SEQS_MAX, kv_heads=512, head_dim=32)   # 2^24 (sequence, head) pairs
    q = fake_queries(total=40000, heads=512, ld=512 * 32)
    assert lib.tav2_kv_attend(ctypes.byref(wide), 0, ctypes.byref(q), 0, FAKE, FAKE, FAKE, 1 << 50,
                              None) == -4
    assert lib.tav2_kv_append(ctypes.byref(wide), 0, FAKE, 512 * 32, FAKE, 512 * 32, FAKE, 200,
                              None) == -4
    for kw in (dict(num_requests=1 << 30, heads=1 << 14, kv_heads=1 << 14, max_len=1 << 27,
                    q_ld=1 << 20, k_ld=1 << 20, v_ld=1 << 20), dict(num_requests=1 << 23)):
        a = fake_window(**kw)
        assert lib.tav2_attend_window(ctypes.byref(a), None) == -4


def test_an_estimate_past_the_tables_divides_as_the_tables_do():
    lib, q = T.load_library(), fake_queries()
    need = [lib.tav2_kv_attend_workspace(ctypes.byref(fake_kv(max_len=n)), ctypes.byref(q))
            for n in (16 * 64 + 63, 16 * 64 + 64, 1 << 20, (1 << 31) - 1)]
    assert need[0] > 0 and need == [need[0]] * 4


# ------------------------------------------------------------------------- the binding
def host_cache(**kw):
    a = dict(layers=1, pages=4, seqs=2, max_blocks=3, kv_heads=2, head_dim=32, device="cpu")
    return T.KvCache.create(**{**a, **kw})


def test_binding_refuses_wrong_shapes_and_types():
    c = host_cache()
    assert c.max_len == 3 * 64 + 63 and c.seqs == 2
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)   # noqa: E731
    i64 = lambda n: torch.zeros(n, dtype=torch.int64)      # noqa: E731
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)      # noqa: E731
    bad = [
        lambda: T.kv_extend(c, i32(3)), lambda: T.kv_extend(c, i64(2)),
        lambda: T.kv_extend(c, torch.zeros(4, dtype=torch.int32)[::2]),
        lambda: T.kv_append(c, 0, bf(5, 2, 32), bf(5, 2, 64), i64(2), 5),
        lambda: T.kv_append(c, 0, bf(5, 3, 32), bf(5, 3, 32), i64(2), 5),
        lambda: T.kv_append(c, 0, bf(5, 2, 32).float(), bf(5, 2, 32), i64(2), 5),
        lambda: T.kv_append(c, 0, bf(5, 2, 32), bf(5, 2, 32), i64(1), 5),
        lambda: T.kv_append(c, 0, bf(5, 32, 2).transpose(1, 2), bf(5, 2, 32), i64(2), 5),
        lambda: T.kv_attend(c, 0, bf(5, 2, 64), i64(3), 5),
        lambda: T.kv_attend(c, 0, bf(5, 2, 32), i64(2), 5),
        lambda: T.kv_attend(c, 0, bf(5, 2, 32), i64(3), 5, out=bf(5, 2, 32).float()),
        lambda: T.kv_attend(c, 0, bf(5, 2, 32), i64(3), 5, lse=torch.zeros(5, 3)),
        lambda: T.kv_fork(c, i32(1)), lambda: T.kv_free(c, i32(2)),
        lambda: T.kv_compact(c, used=i64(1)),
        lambda: T.attend_window(bf(5, 2, 32), bf(4, 2, 32), bf(4, 2, 32), i64(1), i32(1), 5),
        lambda: T.attend_window(bf(5, 2, 32), bf(5, 2, 32), bf(5, 1, 32), i64(1), i32(1), 5),
        lambda: T.attend_window(bf(5, 2, 32), bf(5, 2, 32), bf(5, 2, 32), i64(1), i32(2), 5),
        lambda: T.attend_window(bf(5, 2, 32), bf(5, 2, 32).float(), bf(5, 2, 32), i64(1), i32(1), 5),
        # right in everything but that the tensors are not on a GPU
        lambda: T.kv_extend(c, i32(2)), lambda: T.kv_trim(c, 5),
        lambda: T.kv_attend(c, 0, bf(5, 2, 32), i64(3), 5),
        lambda: T.attend_window(bf(5, 2, 32), bf(5, 2, 32), bf(5, 2, 32), i64(1), i32(1), 5),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted:", i)


def test_append_refuses_fewer_values_than_keys():
    """(kv_append reads offset[s] + i rows of both.)"""
    c = host_cache()
    kv = [torch.zeros(n, 2, 32, dtype=torch.bfloat16) for n in (5, 4)]
    for k, v in ((0, 1), (1, 0)):
        with pytest.raises(ValueError, match="k, v"):
            T.kv_append(c, 0, kv[k], kv[v], torch.zeros(2, dtype=torch.int64), 5)


def test_binding_refuses_a_stream_of_another_device():
    with pytest.raises(ValueError, match="stream"):
        T._run("tav2_kv_trim", 0, SimpleNamespace(device_index=1, cuda_stream=0), ())


def test_binding_refuses_numbers_that_the_abi_does_not_hold(monkeypatch):
    """A window of 2^32 + 5 would be one of 5, sinks of 2^32 none, a scale of 1e-50 the default one."""
    c = host_cache()
    bf, i64, i32 = torch.zeros(5, 2, 32, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64), torch.zeros(
        3, dtype=torch.int32)
    monkeypatch.setattr(T, "_run", lambda *a, **k: None)
    calls = {"window": lambda **k: T.attend_window(bf, bf, bf, i64, i32, **{"max_len": 5, **k}),
             "append": lambda **k: T.kv_append(c, **{"layer": 0, "k": bf, "v": bf, "offset": i64, "max_count": 5, **k}),
             "attend": lambda **k: T.kv_attend(c, **{"layer": 0, "q": bf, "offset": i64, "max_count": 5, **k}),
             "trim": lambda **k: T.kv_trim(c, **{"window": 5, **k}),
             "max_len": lambda max_len: setattr(c, "max_len", max_len)}
    for name, what in (("window", ("max_len", "window", "sinks")), ("append", ("layer", "max_count")),
                       ("attend", ("layer", "max_count", "window", "sinks")), ("trim", ("window", "sinks")),
                       ("max_len", ("max_len",))):
        for key in what:
            calls[name](**{key: 2 ** 31 - 1 if key != "max_count" else 5})
            for bad in (2 ** 32 + 5, 2 ** 32, 2 ** 31, -2 ** 31 - 1):
                with pytest.raises(ValueError, match="32 bits"):
                    calls[name](**{key: bad})
    for name in ("window", "attend"):
        calls[name](scale=1e-44)
        for bad in (1e-50, -1e-60):
            with pytest.raises(ValueError, match="scale"):
                calls[name](scale=bad)


def test_workspace_keeps_what_a_graph_writes_to(monkeypatch):
    """A buffer used in a capture outlives the workspace's growth: replays write to its address.  Others
    are given back."""
    ws = T.Workspace("cpu")
    ws.gpu, capturing = True, [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    ws.get(1000)
    first = weakref.ref(ws.buf)
    capturing[0] = True
    ws.get(500)
    capturing[0] = False
    ws.get(800)
    ws.get(5000)
    second = weakref.ref(ws.buf)
    ws.get(50000)
    assert first() is not None and second() is None and ws.buf.numel() >= 50000


def test_cache_refuses_buffers_that_do_not_fit_together():
    good = host_cache()
    names = ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "table", "length", "fresh", "refs")
    parts = {n: getattr(good, n) for n in names}
    T.KvCache(**parts, max_len=10)
    for n in names:
        for wrong in (parts[n][..., :-1], parts[n].double()):
            with pytest.raises(ValueError):
                T.KvCache(**{**parts, n: wrong}, max_len=10)


# ------------------------------------------------------------------------- the oracle
@pytest.mark.parametrize("L,window,sinks", [(1, 0, 0), (7, 0, 0), (9, 1, 0), (12, 4, 0), (12, 4, 2),
                                            (12, 4, 30), (5, 9, 1)])
def test_oracle_attention_by_loops(L, window, sinks):
    g = np.random.default_rng(L * 100 + window * 10 + sinks)
    q, k, v = g.normal(size=(L, 4, 3)), g.normal(size=(L, 2, 3)), g.normal(size=(L, 2, 3))
    out, lse, size, reach = history.window_attention(q, k, v, window, sinks)
    for p in range(L):
        for h in range(4):
            terms = [(math.fsum(q[p, h] * k[j, h // 2]) / math.sqrt(3), v[j, h // 2]) for j in range(L)
                     if j <= p and (window == 0 or p - j < window or j < sinks)]
            z = math.fsum(math.exp(s) for s, _ in terms)
            want = sum(math.exp(s) / z * x for s, x in terms)
            assert np.allclose(out[p, h], want, rtol=1e-12, atol=1e-13)
            assert np.allclose(size[p, h], sum(math.exp(s) / z * abs(x) for s, x in terms))
            assert math.isclose(lse[p, h], math.log(z), rel_tol=1e-12, abs_tol=1e-12)


def test_oracle_nothing_seen():
    out, lse, _, _ = history.attend(np.ones((2, 1, 4)), np.ones((3, 1, 4)), np.ones((3, 1, 4)),
                                    np.zeros((2, 3), dtype=bool))
    assert (out == 0).all() and (lse == -np.inf).all()


def test_oracle_quantise_is_exact_rounding():
    g = np.random.default_rng(5)
    for trial in range(20):
        x = torch.from_numpy(g.normal(size=(64, 2)) * 10.0 ** g.integers(-3, 4)).bfloat16()
        if trial % 2:   # many exact halves: a largest magnitude of 254 steps
            x = torch.from_numpy(g.integers(-254, 255, size=(64, 2))).bfloat16()
            x[0, 0] = 254
        x = x.double().numpy()
        codes, scale = history.quantise(x)
        top = max(Fraction(float(abs(e))) for e in x.flat)
        for e, c in zip(x.flat, codes.flat):
            assert c == round(Fraction(float(e)) * 127 / top)   # Python rounds halves to even
        assert np.abs(codes).max() == 127
        assert np.abs(codes * scale - x).max() <= scale / 2 * (1 + 1e-9)
    assert history.quantise(np.zeros((64, 2)))[1] == 1.0
    assert (history.quantise(np.full((64, 2), 2.0 ** -101))[0] == 0).all()


def test_oracle_cache_pages():
    c = history.Cache(seqs=4, pages=6, max_blocks=3)
    c.extend([130, 63, 0, 64])
    assert c.table == [[0, 1], [], [], [2]] and c.fresh == [130, 63, 0, 64]
    c.extend([0, 1, 300, 0])          # 300 tokens pass max_blocks
    assert c.table[1] == [3] and c.fresh == [0, 1, 0, 0] and c.len == [130, 64, 0, 64]
    c.extend([62, 128, 0, 1])         # one page for the first, none of two for the second: none behind
    assert c.table[0] == [0, 1, 4] and c.fresh == [62, 0, 0, 0] and c.len[3] == 64
    for s in range(4):
        c.k[s] = c.v[s] = [np.zeros((1, 1, 1))] * c.len[s]
    c.fork([-1, -1, 0, 1])            # the last is not empty
    assert c.table[2] == [0, 1, 4] and c.refs == [2, 2, 1, 1, 2, 0]
    c.free([1, 1, 0, 0])
    assert c.refs == [1, 1, 1, 0, 1, 0] and c.len == [0, 0, 192, 64]
    c.trim(window=65, sinks=1)        # of 192 tokens the last 64 and the first stay
    assert c.table[2] == [0, None, 4] and c.refs == [1, 0, 1, 0, 1, 0] and c.table[3] == [2]
    assert c.compact() == 3
    assert c.table[2] == [0, None, 1] and c.refs == [1, 1, 1, 0, 0, 0]
