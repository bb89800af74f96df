"""Host side of the calls on held tokens (chunk attention, weights, eviction): refusals and sizes, nothing is launched; and the plain eviction."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
from paper_2603_04460_amd import binding
from plain_held import stays


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 4096)()
    yield (ctypes.addressof(buf) + 15) & ~15
    del buf


def cache(p, **kw):
    x = dict(data=p, pages=8, kv_heads=2, page_size=64, table=p, max_pages=4)
    x.update(kw)
    return binding._Cache(x["data"], x["pages"], x["kv_heads"], x["page_size"], x["table"], x["max_pages"])


BAD_CACHE = [(dict(data=None), -1), (dict(data=8), -1), (dict(pages=0), -1), (dict(kv_heads=0), -1), (dict(page_size=0), -1), (dict(page_size=96), -2),
             (dict(page_size=32), -2), (dict(table=2), -1), (dict(max_pages=0), -1), (dict(max_pages=1), -1), (dict(kv_heads=4097), -2),
             (dict(pages=1 << 31), -2), (dict(table=None, pages=7), -1)]
HUGE = 1 << 62


def at(p, kw):
    return {k: p + v if k in ("data", "table") and v in (2, 8) else v for k, v in kw.items()}


def test_prefill_refused(p):
    L = binding._load()

    def call(c=None, q=p, batch=2, hq=4, rows=200, lens=p, n=256, scale=0.1, o=p, lse=p, ws=p, size=HUGE):
        c = cache(p) if c is None else c
        return L.vs_cache_prefill(q, ctypes.byref(c), batch, hq, rows, lens, n, scale, o, lse, ws, size, None)

    for kw, code in BAD_CACHE:
        assert call(cache(p, **at(p, kw))) == code, kw
    assert L.vs_cache_prefill(p, None, 1, 4, 200, p, 100, 0.1, p, p, p, HUGE, None) == -1
    for kw, code in ((dict(q=None), -1), (dict(q=p + 8), -1), (dict(o=None), -1), (dict(o=p + 4), -1), (dict(lse=p + 8), -1), (dict(ws=p + 8), -1), (dict(batch=0), -1),
                     (dict(hq=0), -1), (dict(rows=0), -1), (dict(rows=-1), -1), (dict(lens=p + 1), -1), (dict(n=0), -1), (dict(n=257), -1), (dict(scale=0.0), -1),
                     (dict(scale=-1.0), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(scale=3e38), -1), (dict(hq=3), -2), (dict(hq=4098), -2),
                     (dict(batch=65536), -2), (dict(rows=(1 << 20) + 1), -2), (dict(rows=1 << 62), -2), (dict(n=(1 << 20) + 1), -2)):
        assert call(**kw) == code, kw
    big = cache(p, kv_heads=8, max_pages=2048, pages=2048)
    need = vs.cache_prefill_workspace(1, 32, 8, 300, 131072)
    for size, ws in ((need - 1, p), (0, None), (need, None)):
        if need and size < need or ws is None and need:
            assert call(big, batch=1, hq=32, rows=300, n=131072, ws=ws, size=size) == -3


@pytest.mark.parametrize("rows", [1, 17, 128])
def test_prefill_of_few_rows_is_the_call_for_few_rows(p, rows):
    for n in (100, 3000):
        assert vs.cache_prefill_workspace(3, 8, 2, rows, n) == vs.cache_attend_workspace(3, 8, 2, rows, n)
    L = binding._load()
    c = ctypes.byref(cache(p))
    assert L.vs_cache_prefill(p, c, 1, 3, rows, p, 100, 0.1, p, None, p, HUGE, None) == -2
    assert L.vs_cache_prefill(p, c, 1, 4, rows, p, 257, 0.1, p, None, p, HUGE, None) == -1


@pytest.mark.parametrize("batch, hq, hk, rows", [(1, 32, 8, 128), (16, 32, 8, 40), (5, 12, 6, 65), (2, 8, 8, 128), (1, 4096, 1, 33)])
def test_prefill_workspace_is_enough_for_smaller_max_n(batch, hq, hk, rows):
    """Where long sequences go to one kernel and short ones to the other."""
    most = 0
    for n in (1, 63, 64, 500, 2000, 4096, 4097, 8000, 16000, 24576, 40000, 131072, 1 << 20):
        need = vs.cache_prefill_workspace(batch, hq, hk, rows, n)
        assert need >= most and need >= vs.cache_attend_workspace(batch, hq, hk, rows, n)
        most = need


def test_workspaces_are_enough_for_smaller_max_n():
    rng = random.Random(3)
    for _ in range(400):
        hk = rng.choice([1, 2, 8])
        sizes = rng.choice([1, 1, 2, 5, 60]), hk * rng.choice([1, 2, 4, 8]), hk, rng.randint(1, rng.choice([40, 300, 4000]))
        n = rng.randint(1, 20000)
        for f in (vs.cache_prefill_workspace, vs.cache_weigh_workspace):
            assert f(*sizes, rng.randint(1, n)) <= f(*sizes, n), (f.__name__, sizes, n)


@pytest.mark.parametrize("rows", [100, 128])
def test_prefill_of_few_rows_of_long_sequences_refused(p, rows):
    """Rows for which vs_cache_prefill takes its own kernel, like any others."""
    L = binding._load()
    c = cache(p, kv_heads=8, max_pages=2048, pages=2048)
    need = vs.cache_prefill_workspace(1, 32, 8, rows, 131072)
    assert need > vs.cache_attend_workspace(1, 32, 8, rows, 131072)

    def call(q=p, hq=32, o=p, ws=p, size=HUGE, scale=0.1, lens=p, n=131072):
        return L.vs_cache_prefill(q, ctypes.byref(c), 1, hq, rows, lens, n, scale, o, p, ws, size, None)

    for kw, code in ((dict(q=None), -1), (dict(o=p + 4), -1), (dict(lens=p + 2), -1), (dict(n=131073), -1), (dict(scale=0.0), -1), (dict(hq=33), -2),
                     (dict(size=need - 1), -3), (dict(ws=None), -3)):
        assert call(**kw) == code, kw


def test_weigh_refused(p):
    L = binding._load()

    def call(c=None, q=p, lse=p, batch=2, hq=4, rows=3, lens=p, n=256, scale=0.1, old=p, decay=1.0, fresh=3, w=p, stride=256, ws=p, size=HUGE):
        c = cache(p) if c is None else c
        return L.vs_cache_weigh(q, lse, ctypes.byref(c), batch, hq, rows, lens, n, scale, old, decay, fresh, w, stride, ws, size, None)

    for kw, code in BAD_CACHE:
        assert call(cache(p, **at(p, kw))) == code, kw
    assert L.vs_cache_weigh(p, p, None, 1, 4, 1, p, 100, 0.1, p, 1.0, 1, p, 100, p, HUGE, None) == -1
    for kw, code in ((dict(q=None), -1), (dict(q=p + 8), -1), (dict(lse=None), -1), (dict(lse=p + 4), -1), (dict(w=None), -1), (dict(w=p + 2), -1), (dict(old=p + 1), -1),
                     (dict(ws=p + 8), -1), (dict(batch=0), -1), (dict(hq=0), -1), (dict(rows=0), -1), (dict(lens=p + 1), -1), (dict(n=0), -1), (dict(n=257), -1),
                     (dict(scale=0.0), -1), (dict(scale=math.nan), -1), (dict(scale=3e38), -1), (dict(scale=1e-39), -1), (dict(decay=-0.1), -1), (dict(decay=1.1), -1),
                     (dict(decay=math.nan), -1), (dict(fresh=-1), -1), (dict(stride=255), -1), (dict(stride=1 << 62), -1), (dict(hq=3), -2), (dict(hq=4098), -2),
                     (dict(batch=65536), -2), (dict(rows=(1 << 20) + 1), -2), (dict(n=(1 << 20) + 1), -2)):
        assert call(**kw) == code, kw
    many = cache(p, kv_heads=1, max_pages=1 << 14, pages=1 << 20)
    assert call(many, batch=1, hq=4096, rows=1 << 20, n=1 << 20, stride=1 << 20) == -2
    need = vs.cache_weigh_workspace(1, 32, 8, 4096, 2000)
    if need:
        assert call(cache(p, kv_heads=8, max_pages=40, pages=40), batch=1, hq=32, rows=4096, n=2000, stride=2000, size=need - 1) == -3


def test_evict_refused(p):
    L = binding._load()

    def call(c=None, w=p, stride=256, batch=2, lens=p, n=256, keep=100, sink=4, recent=10, to=None, out=p, stride_out=256, kept=p, after=p, ws=p, size=HUGE):
        c = cache(p) if c is None else c
        return L.vs_cache_evict(ctypes.byref(c), w, stride, batch, lens, n, keep, sink, recent, None if to is None else ctypes.byref(to), out, stride_out, kept, after,
                                ws, size, None)

    for kw, code in BAD_CACHE:
        assert call(cache(p, **at(p, kw))) == code, kw
        if kw != dict(max_pages=1):
            assert call(to=cache(p, **at(p, kw))) == code, kw
    assert L.vs_cache_evict(None, p, 256, 1, p, 256, 100, 0, 0, None, None, 0, None, p, p, HUGE, None) == -1
    for kw, code in ((dict(w=None), -1), (dict(w=p + 2), -1), (dict(out=p + 1), -1), (dict(kept=p + 3), -1), (dict(after=None), -1), (dict(after=p + 2), -1), (dict(ws=p + 4), -1),
                     (dict(lens=p + 1), -1), (dict(batch=0), -1), (dict(n=0), -1), (dict(n=257), -1), (dict(keep=0), -1), (dict(keep=-1), -1), (dict(sink=-1), -1),
                     (dict(recent=-1), -1), (dict(sink=91), -1), (dict(sink=101, recent=0), -1), (dict(recent=97), -1), (dict(sink=1 << 62, recent=1 << 62), -1),
                     (dict(stride=255), -1), (dict(stride=1 << 62), -1), (dict(stride_out=99), -1), (dict(stride_out=1 << 62), -1), (dict(keep=257, stride_out=300), -1),
                     (dict(to=cache(p, kv_heads=1)), -1), (dict(to=cache(p, max_pages=1)), -1), (dict(keep=(1 << 20) + 1), -2), (dict(batch=65536), -2),
                     (dict(n=(1 << 20) + 1), -2), (dict(ws=None), -3), (dict(size=vs.cache_evict_workspace(2, 2, 256, 100) - 1), -3)):
        assert call(**kw) == code, kw


def test_sizes():
    for f, ok, bad in ((vs.cache_prefill_workspace, (2, 8, 2, 500, 9000), ((0, 8, 2, 500, 9000), (2, 0, 2, 500, 9000), (2, 9, 2, 500, 9000), (2, 8, 2, 0, 9000), (2, 8, 2, 500, 0),
                                                                           (65536, 8, 2, 500, 9000), (40000, 8, 2, 500, 9000), (2, 8, 2, (1 << 20) + 1, 9000), (2, 8, 2, 500, (1 << 20) + 1),
                                                                           (1, 8192, 8192, 500, 9000))),
                       (vs.cache_weigh_workspace, (2, 8, 2, 500, 9000), ((0, 8, 2, 500, 9000), (2, 9, 2, 500, 9000), (2, 8, 2, 0, 9000), (2, 8, 2, 500, (1 << 20) + 1))),
                       (vs.cache_evict_workspace, (2, 2, 9000, 500), ((0, 2, 9000, 500), (2, 0, 9000, 500), (2, 2, 0, 500), (2, 2, 9000, 0), (2, 2, 9000, (1 << 20) + 1),
                                                                      (2, 2, (1 << 20) + 1, 500), (65535, 2, 9000, 500)))):
        assert f(*ok) < 1 << 32
        for x in bad:
            assert f(*x) == 0, x
    assert vs.cache_evict_workspace(2, 2, 9000, 500) >= 4 * (500 * 4 * 2 + 8 * 8704)
    assert vs.cache_evict_workspace(65535, 1, 1 << 20, 1 << 20) > 1 << 32


@pytest.mark.parametrize("batch, hq, hk, n_q", [(1, 32, 8, 129), (1, 1, 1, 500), (4, 8, 2, 2000), (64, 32, 8, 300), (1, 32, 8, 1 << 20), (3, 16, 2, 4000), (1, 4096, 1, 1000)])
def test_workspace_for_the_longest_sequence(batch, hq, hk, n_q):
    lengths = sorted({1 << i for i in range(21)} | {100, 600, 5000, 131000, 1000000})
    for f in (vs.cache_prefill_workspace, vs.cache_weigh_workspace):
        sizes = [f(batch, hq, hk, n_q, n) for n in lengths]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_plain_eviction():
    yes = np.ones(8, dtype=bool)
    w = np.array([1, 5, 2, 5, 0, 3, np.nan, 4], dtype=np.float32)
    assert stays(w, yes, 3, 0, 0) == [1, 3, 7] and stays(w, yes, 4, 1, 1) == [0, 1, 3, 7] and stays(w, yes, 7, 0, 0) == [0, 1, 2, 3, 4, 5, 7]
    assert stays(w, yes, 2, 0, 2) == [6, 7] and stays(w, yes, 9, 0, 0) == list(range(8))
    assert stays(w, np.array([1, 0, 1, 1, 1, 1, 1, 1], dtype=bool), 3, 2, 0) == [0, 3, 7]
    assert stays(np.array([-0.0, 0.0, -np.inf, np.nan], dtype=np.float32), yes[:4], 1, 0, 0) == [0]


def test_binding_refuses(monkeypatch):
    """What the binding checks before the library: devices (host tensors stand for the current one), shapes, types."""
    def dev(t, dtype, what):
        if not (isinstance(t, torch.Tensor) and t.is_contiguous() and t.dtype == dtype):
            raise TypeError(what)
        return t
    monkeypatch.setattr(binding, "_dev", dev)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    data = torch.zeros(8, 2, 1, vs.CACHE_BLOCK_BYTES, dtype=torch.uint8)
    c = vs.Cache(data, torch.zeros(2, 4, dtype=torch.int32))
    q, w = torch.zeros(2, 4, 3, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 256)
    lse, lens = torch.zeros(2, 4, 3), torch.zeros(2, dtype=torch.int32)
    for bad in (dict(lse=lse[:, :, :2].contiguous()), dict(weights=w[:1].contiguous()), dict(old=w[:, :, :100].contiguous()), dict(lens=lens[:1].contiguous()), dict(q=q[:1].contiguous())):
        kw = dict(q=q, lse=lse, weights=w, old=None, lens=lens)
        kw.update(bad)
        with pytest.raises(AssertionError):
            vs.cache_weigh(kw["q"], kw["lse"], c, kw["weights"], 256, lens=kw["lens"], old=kw["old"])
    for bad in (dict(lse=lse.double()), dict(weights=w.half()), dict(old=w.double()), dict(lens=lens.long()), dict(q=q.half()), dict(weights=w[:, :, ::2]), dict(ws=w[:, :, ::2])):
        kw = dict(q=q, lse=lse, weights=w, old=None, lens=lens, ws=None)
        kw.update(bad)
        with pytest.raises(TypeError):
            vs.cache_weigh(kw["q"], kw["lse"], c, kw["weights"], 256, lens=kw["lens"], old=kw["old"], ws=kw["ws"])
    kept = torch.zeros(2, 2, 100, dtype=torch.int32)
    ok = dict(weights=w, lens_out=lens, lens=lens, weights_out=w, kept=kept, to=None, ws=None)
    for bad, error in ((dict(weights=w[:1].contiguous()), AssertionError), (dict(lens=lens[:1].contiguous()), AssertionError), (dict(kept=kept[:, :, :9].contiguous()), AssertionError),
                       (dict(weights_out=w[:1].contiguous()), AssertionError), (dict(lens_out=lens[:1].contiguous()), AssertionError), (dict(kept=kept.long()), TypeError),
                       (dict(weights=w.half()), TypeError), (dict(lens_out=lens.long()), TypeError), (dict(to=vs.Cache(data, torch.zeros(1, 4, dtype=torch.int32))), AssertionError),
                       (dict(ws=w[:, :, ::2]), TypeError)):
        kw = dict(ok)
        kw.update(bad)
        with pytest.raises(error):
            vs.cache_evict(c, kw["weights"], 256, 100, kw["lens_out"], lens=kw["lens"], weights_out=kw["weights_out"], kept=kw["kept"], to=kw["to"], ws=kw["ws"])
    for bad, error in ((dict(q=q.float()), TypeError), (dict(o=q[:1].contiguous()), AssertionError), (dict(lse=lse[:1].contiguous()), AssertionError)):
        kw = dict(q=q, o=q, lse=lse)
        kw.update(bad)
        with pytest.raises(error):
            vs.cache_prefill(kw["q"], c, kw["o"], 256, lse=kw["lse"])
