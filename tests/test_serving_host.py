"""Host side of the calls around the prefill: refusals, sizes, frequencies, and the plain form of the cache that the GPU tests compare with."""
import ctypes
import math

import numpy as np
import pytest

import paper_2603_04460_amd as vs
import plain_serving as plain
from paper_2603_04460_amd import binding

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 4096)()
    yield (ctypes.addressof(buf) + 15) & ~15
    del buf


def cache(p, **kw):
    x = dict(data=p, pages=8, kv_heads=2, page_size=64, table=p, max_pages=4)
    x.update(kw)
    return binding._Cache(x["data"], x["pages"], x["kv_heads"], x["page_size"], x["table"], x["max_pages"])


def test_frequencies():
    for rot in (8, 64, 96, 128):
        base = 5e5 ** (-2.0 * np.arange(rot // 2) / rot)
        # pow and a few products: within 8 roundings of 2^-53
        near = lambda got, want: np.abs(got.numpy() / want - 1).max() <= 8 * 2.0 ** -53
        assert near(vs.rope_frequencies(5e5, rot), base)
        assert near(vs.rope_frequencies(5e5, rot, scaling=1, factor=4.0), base / 4)
        got = vs.rope_frequencies(5e5, rot, scaling=2, factor=8.0, low=1.0, high=4.0, original=8192.0).numpy()
        turns = 8192 * base / (2 * math.pi)
        assert np.array_equal(got[turns >= 4], vs.rope_frequencies(5e5, rot).numpy()[turns >= 4])
        assert np.abs(got[turns <= 1] * 8 / base[turns <= 1] - 1).max(initial=0) <= 8 * 2.0 ** -53
        mid = (turns > 1) & (turns < 4)
        mix = (turns[mid] - 1) / 3
        assert np.abs(got[mid] / (base[mid] * ((1 - mix) / 8 + mix)) - 1).max(initial=0) <= 32 * 2.0 ** -53
        assert (np.diff(got) < 0).all()


def test_frequencies_refused():
    L = binding._load()
    f = (ctypes.c_double * 64)()
    ok = (1e6, 128, 2, 8.0, 1.0, 4.0, 8192.0)
    assert L.vs_rope_frequencies(*ok, f) == 0
    assert L.vs_rope_frequencies(*ok, None) == -1
    for at, bad, code in ((0, 1.0, -1), (0, math.nan, -1), (1, 0, -2), (1, 12, -2), (1, 136, -2), (2, 3, -1), (2, -1, -1), (3, 0.5, -1),
                          (3, math.inf, -1), (4, 0.0, -1), (5, 1.0, -1), (6, 0.0, -1)):
        args = list(ok)
        args[at] = bad
        assert L.vs_rope_frequencies(*args, f) == code, (at, bad)
    assert L.vs_rope_frequencies(1e6, 128, 0, 0.0, 0.0, 0.0, 0.0, f) == 0        # unused arguments are not looked at


def test_norm_rope_refused(p):
    L = binding._load()

    def call(q=(p, 128, 128), k=(p, 128, 128), v=None, batch=1, rows=4, hq=2, hk=1, w=p, eps=1e-6, freq=p, rot=128, pairing=0, mag=1.0,
             lens=None, pos0=0, qo=p, ko=p, vo=None):
        x = [None if r is None else binding._Rows(*r) for r in (q, k, v)]
        ref = [None if r is None else ctypes.byref(r) for r in x]
        t = binding._Rotation(freq, rot, pairing, mag)
        return L.vs_qk_norm_rope(*ref, batch, rows, hq, hk, w, w, eps, ctypes.byref(t), lens, pos0, qo, ko, vo, None)

    for bad in (dict(q=None), dict(k=None), dict(q=(None, 128, 128)), dict(q=(p + 4, 128, 128)), dict(q=(p, 127, 128)), dict(k=(p, 128, 132)),
                dict(k=(p, 64, 128)), dict(v=(p, 128, 128)), dict(vo=p), dict(batch=0), dict(rows=0), dict(hq=0), dict(hk=-1), dict(w=p + 4),
                dict(eps=0.0), dict(eps=math.nan), dict(freq=None), dict(freq=p + 8), dict(pairing=2), dict(mag=math.inf), dict(lens=p + 2),
                dict(pos0=-1), dict(qo=None), dict(ko=p + 8)):
        assert call(**bad) == -1, bad
    for bad in (dict(rot=0), dict(rot=4), dict(rot=100), dict(rot=136), dict(rows=(1 << 20) + 1), dict(batch=65536), dict(batch=65535, rows=1 << 20)):
        assert call(**bad) == -2, bad
    assert L.vs_qk_norm_rope(ctypes.byref(binding._Rows(p, 128, 128)), ctypes.byref(binding._Rows(p, 128, 128)), None, 1, 1, 1, 1, None, None,
                             0.0, None, None, 0, p, p, None, None) == -1


def test_cache_refused(p):
    L = binding._load()
    bad_cache = [(dict(data=None), -1), (dict(data=p + 8), -1), (dict(pages=0), -1), (dict(kv_heads=0), -1), (dict(page_size=0), -1),
                 (dict(page_size=96), -2), (dict(page_size=32), -2), (dict(table=p + 2), -1), (dict(max_pages=0), -1), (dict(max_pages=1), -1),
                 (dict(kv_heads=4097), -2), (dict(pages=1 << 31), -2), (dict(table=None, pages=7), -1)]
    calls = {
        "write": lambda c, k=p, v=p, batch=2, rows=3, lens=p, n=100: L.vs_cache_write(c, k, v, batch, rows, lens, n, None),
        "read": lambda c, k=p, v=p, batch=2, rows=3, lens=p, n=100: L.vs_cache_read(c, batch, rows, lens, n, k, v, None),
        "attend": lambda c, k=p, v=p, batch=2, rows=3, lens=p, n=100: L.vs_cache_attend(k, c, batch, 4, rows, lens, n, 0.1, v, None, p, 1 << 20, None),
    }
    for name, call in calls.items():
        for kw, code in bad_cache:
            x = cache(p, **kw)
            assert call(ctypes.byref(x)) == code, (name, kw)
        x = ctypes.byref(cache(p))
        assert call(None) == -1
        for kw, code in ((dict(k=p + 8), -1), (dict(v=p + 4), -1), (dict(batch=0), -1), (dict(rows=0), -1), (dict(lens=p + 1), -1), (dict(n=0), -1),
                         (dict(n=257), -1), (dict(batch=65536), -2), (dict(rows=(1 << 20) + 1), -2)):
            assert call(x, **kw) == code, (name, kw)
    x = ctypes.byref(cache(p))
    assert calls["write"](x, k=None) == -1 and calls["write"](x, v=None) == -1 and calls["read"](x, k=None, v=None) == -1
    long = ctypes.byref(cache(p, page_size=64, max_pages=1 << 20, pages=1 << 24))
    assert calls["write"](long, n=(1 << 20) + 1) == -2
    attend = lambda hq=4, rows=3, scale=0.1, o=p, lse=None, ws=p, size=1 << 20, n=100, c=x: L.vs_cache_attend(p, c, 2, hq, rows, None, n, scale, o, lse,
                                                                                                              ws, size, None)
    assert attend(hq=0) == -1 and attend(hq=3) == -2 and attend(hq=4100) == -2 and attend(rows=129) == -2 and attend(o=None) == -1
    assert attend(scale=0.0) == -1 and attend(scale=math.nan) == -1 and attend(scale=math.inf) == -1 and attend(lse=p + 8) == -1
    need = vs.cache_attend_workspace(2, 4, 2, 3, 100000)
    assert need > 0
    long = ctypes.byref(cache(p, max_pages=2000, pages=4000))
    assert attend(ws=None, size=0, n=100000, c=long) == -3 and attend(size=need - 1, n=100000, c=long) == -3
    assert attend(ws=p + 8, size=need, n=100000, c=long) == -1


def test_sizes():
    assert vs.cache_bytes(10, 8, 256) == 10 * 8 * 4 * vs.CACHE_BLOCK_BYTES and vs.CACHE_BLOCK_BYTES == 64 * 136
    assert vs.cache_bytes(0, 8, 64) == vs.cache_bytes(1, 0, 64) == vs.cache_bytes(1, 1, 63) == vs.cache_bytes(1, 1, 96) == 0
    assert vs.cache_bytes(1 << 20, 8, 1024) == (1 << 20) * 8 * 16 * 8704            # past 32 bits
    assert vs.cache_attend_workspace(1, 3, 2, 1, 100) == vs.cache_attend_workspace(1, 4, 2, 129, 100) == vs.cache_attend_workspace(0, 4, 2, 1, 100) == 0


@pytest.mark.parametrize("batch, hq, hk, n_q", [(1, 32, 8, 1), (1, 1, 1, 1), (4, 8, 2, 5), (64, 32, 8, 1), (1, 32, 8, 128), (3, 16, 2, 7)])
def test_workspace_for_the_longest_sequence(batch, hq, hk, n_q):
    sizes = [vs.cache_attend_workspace(batch, hq, hk, n_q, n) for n in sorted({1 << i for i in range(21)} | {100, 600, 5000, 131000, 1000000})]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("hq, n_q", [(150, 128), (256, 64), (513, 128), (4096, 128)])
def test_workspace_of_ten_thousand_rows(hq, n_q):
    """So many rows that a workgroup's share of them is all of the call: the largest sequence's workspace serves the shorter ones, too."""
    sizes = [vs.cache_attend_workspace(1, hq, 1, n_q, n) for n in sorted({1 << i for i in range(21)} | {600, 2000, 2300, 5000, 12345, 131000})]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[-1] > 0


def test_largest_calls(p):
    """Sizes behind which a launch or a value would leave 32 bits are refused, whatever memory there is."""
    L = binding._load()
    many = ctypes.byref(cache(p, kv_heads=1, max_pages=4, pages=1 << 20, table=p))
    attend = lambda batch, hq, n_q, scale=0.1: L.vs_cache_attend(p, many, batch, hq, n_q, None, 100, scale, p, None, p, 1 << 60, None)
    assert attend(32, 4096, 128) == -2 and attend(1 << 12, 32, 128) == -2
    assert attend(1, 1, 1, scale=3e38) == -1                # scale * log2(e) is past fp32
    t = binding._Rotation(p, 128, 0, 1.0)
    x = ctypes.byref(binding._Rows(p, 128, 128))
    norm = lambda eps=1e-6, pos0=0, rows=4: L.vs_qk_norm_rope(x, x, None, 1, rows, 1, 1, p, p, eps, ctypes.byref(t), None, pos0, p, p, None, None)
    assert norm(pos0=(1 << 31) - 3) == -2 and norm(pos0=1 << 62) == -2
    assert norm(eps=1e-39) == -1 and norm(eps=1.5) == -1


def test_plain_cache():
    """The plain form itself: its codes stand for the nearest numbers, a block's bytes hold every token once."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((64, 128)) * 10.0 ** rng.integers(-3, 4, (64, 1))
    code, e = plain.quantise(x)
    y = plain.values(code, e)
    s = 2.0 ** (np.repeat(e, 32, -1).reshape(64, 128).astype(float) - 127)
    assert (np.abs(x) <= 7 * s).all() and (np.abs(x).reshape(64, 4, 32).max(-1) > 3.5 * s.reshape(64, 4, 32)[..., 0]).all()
    assert (np.abs(x - y) <= s).all()                       # half of the widest step
    assert np.array_equal(*[plain.values(*plain.quantise(z)) for z in (y, x)])      # what the cache holds stays as it is
    tie = np.zeros(128)
    tie[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]
    assert plain.values(*plain.quantise(tie))[:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    seen = np.zeros((plain.BLOCK_BYTES, 2), dtype=int)
    for t in range(64):
        for ch in range(128):
            at, high = plain.v_place(ch, t)
            seen[at, high] += 1
    assert (seen[4096:8192] == 1).all() and seen[:4096].sum() == 0
    for marked in (0, 1):                                   # every byte of a block belongs to a token
        block = np.full(plain.BLOCK_BYTES, 0xff * marked, dtype=np.uint8)
        for t in range(64):
            plain.put(block, t, np.full(128, 5), np.full(4, 9), np.full(128, 6), np.full(4, 8))
        assert set(block[:4096]) == {0x55} and set(block[4096:8192]) == {0x66} and set(block[8192:8448]) == {9} and set(block[8448:]) == {8}
