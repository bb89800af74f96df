"""Weights of held tokens against the plain form in 64 bits; how far they may be off is derived there."""
import pytest
import torch

import paper_2603_04460_amd as vs
from plain_held import attention, filled, ints, kv, normal, weights

pytestmark = pytest.mark.gpu


def inputs(seed, hq, hk, rows, lens, page=64, n=None):
    """A cache, queries, and the lse that an attention of them leaves (the plain one's, rounded)."""
    batch, n = len(lens), n or max(lens)
    k, v = kv(seed, batch, hk, n)
    cache = filled(seed, k, v, page)
    q = normal(seed + 7, batch, hq, rows, 128).bfloat16().cuda()
    return cache, q, attention(q, cache, lens, n)[1].float().cuda()


def call(q, lse, cache, lens, max_n, old=None, decay=1.0, fresh=None, stride=None, scale=None):
    batch, hq, rows, _ = q.shape
    out = torch.full((batch, cache.kv_heads, stride or max_n), 7.0, device="cuda")
    ws = torch.full((vs.cache_weigh_workspace(batch, hq, cache.kv_heads, rows, max_n),), 0xff, dtype=torch.uint8, device="cuda")
    vs.cache_weigh(q, lse, cache, out, max_n, lens=None if lens is None else ints(*lens), old=old, decay=decay, fresh=fresh, ws=ws, scale=scale)
    return out


def near(got, want, lens):
    w, tol = want
    got = got.double().cpu()
    for b, n in enumerate(lens):
        n = max(n, 0)
        assert (got[b, :, n:] == 7.0).all()
        x, y = got[b, :, :n], w[b, :, :n]
        assert torch.equal(torch.isnan(x), torch.isnan(y))
        worst = ((x - y).abs() - tol[b, :, :n])[torch.isfinite(y)]
        assert worst.numel() == 0 or worst.max() <= 0, (worst.max(), (x - y).abs().max())


@pytest.mark.parametrize("hq, hk", [(1, 1), (4, 1), (8, 2), (3, 3), (16, 2), (6, 2), (64, 1)])
@pytest.mark.parametrize("rows, lens", [(1, [1, 700, 0, 64, 65]), (2, [1, 100, 0, 2]), (5, [4, 513, 0]), (33, [300, 20]), (200, [700, 0, 150])])
def test_heads_and_lengths(hq, hk, rows, lens):
    cache, q, lse = inputs(rows + hq, hq, hk, rows, lens)
    n = max(lens)
    old = torch.rand(len(lens), hk, n, generator=torch.Generator().manual_seed(3)).cuda()
    near(call(q, lse, cache, lens, n, old=old), weights(q, lse, cache, lens, n, old, 1.0, rows), lens)


@pytest.mark.parametrize("page", [64, 192, 1024])
@pytest.mark.parametrize("n, rows", [(4001, 1), (4096, 16), (2000, 300), (1111, 1111), (20000, 4)])
def test_pages(page, n, rows):
    cache, q, lse = inputs(n, 8, 2, rows, [n], page)
    near(call(q, lse, cache, [n], n), weights(q, lse, cache, [n], n, None, 1.0, rows), [n])


@pytest.mark.parametrize("hq, hk, rows, n", [(8, 2, 20, 131072), (8, 8, 17, 280000)])
def test_many_groups_of_a_workgroup(hq, hk, rows, n):
    """Long sequences whose few tiles of rows stay in LDS for several groups of keys."""
    cache, q, lse = inputs(61, hq, hk, rows, [n], 256)
    near(call(q, lse, cache, [n], n), weights(q, lse, cache, [n], n, None, 1.0, rows), [n])


@pytest.mark.parametrize("rows", [1, 7, 40])
def test_sum_of_a_row_is_one(rows):
    """What the rows of a head give away is as much as there are rows that see something."""
    lens = [900, 3, 0, 64]
    cache, q, lse = inputs(11, 8, 2, rows, lens)
    got = call(q, lse, cache, lens, 900).double().cpu()
    for b, n in enumerate(lens):
        # (each exponent is off by no more than 2^-17 of the sum of its terms, here below 60)
        assert (got[b, :, :n].sum(-1) - 4 * min(rows, n)).abs().max() <= 4 * rows * 60 * 2.0 ** -17


@pytest.mark.parametrize("decay, fresh", [(1.0, 0), (0.5, 3), (0.0, 0), (0.9, 10 ** 6), (0.25, 120)])
def test_old_weights(decay, fresh):
    """Decayed, but for the tokens that have none yet, whatever stands there."""
    lens = [500, 90, 0]
    cache, q, lse = inputs(13, 4, 1, 2, lens)
    old = torch.rand(3, 1, 500, generator=torch.Generator().manual_seed(5)).cuda()
    for b, n in enumerate(lens):
        old[b, :, max(0, n - fresh):] = float("nan")
    if decay == 0.0:
        old[:] = float("nan")
    near(call(q, lse, cache, lens, 500, old=old, decay=decay, fresh=fresh), weights(q, lse, cache, lens, 500, old, decay, fresh), lens)


def test_in_place():
    """old is weights, with rows further apart than max_n."""
    lens = [300, 301]
    cache, q, lse = inputs(15, 4, 2, 1, lens)
    w = torch.rand(2, 2, 333, generator=torch.Generator().manual_seed(7)).cuda()
    old = w.clone()
    vs.cache_weigh(q, lse, cache, w, 301, lens=ints(*lens), old=w, decay=0.75)
    want, tol = weights(q, lse, cache, lens, 301, old, 0.75, 1)
    for b, n in enumerate(lens):
        assert torch.equal(w[b, :, n:], old[b, :, n:])
        assert ((w[b, :, :n].double().cpu() - want[b, :, :n]).abs() <= tol[b, :, :n]).all()


def test_lengths_of_the_host():
    cache, q, lse = inputs(17, 4, 2, 3, [400, 400])
    want = call(q, lse, cache, [400, 400], 400)
    assert torch.equal(call(q, lse, cache, None, 400), want) and torch.equal(call(q, lse, cache, [5000, 400], 400), want)
    assert torch.equal(call(q, lse, cache, [400, 400], 400, stride=600)[:, :, :400], want)
    none = call(q, lse, cache, [-1, 400], 400)
    assert (none[0] == 7.0).all() and torch.equal(none[1], want[1])


def test_missing_pages():
    """A token without a page gets nothing and keeps what it had."""
    lens = [640, 640]
    k, v = kv(19, 2, 2, 640)
    cache = filled(19, k, v, 128)
    t = cache.table.clone()
    t[0, 1], t[1, 0], t[1, 4] = -1, cache.pages, 2 ** 31 - 1
    cache.table = t
    q = normal(20, 2, 4, 3, 128).bfloat16().cuda()
    lse = attention(q, cache, lens, 640)[1].float().cuda()
    old = torch.rand(2, 2, 640, generator=torch.Generator().manual_seed(9)).cuda()
    got = call(q, lse, cache, lens, 640, old=old, decay=0.5)
    near(got, weights(q, lse, cache, lens, 640, old, 0.5, 3), lens)
    assert torch.equal(got[0, :, 128:256], old[0, :, 128:256] * 0.5)


def test_rows_without_a_key_and_what_is_not_finite():
    """lse of -inf adds nothing, +inf neither; NaN reaches the keys that its row sees; a key that is not finite is not a number itself."""
    n, rows = 200, 40
    cache, q, lse = inputs(21, 2, 1, rows, [n])
    lse[0, 0, 3], lse[0, 1, 30] = -float("inf"), float("inf")
    near(call(q, lse, cache, [n], n), weights(q, lse, cache, [n], n, None, 1.0, rows), [n])
    lse[0, 1, 20] = float("nan")
    got = call(q, lse, cache, [n], n)
    assert torch.isnan(got[0, 0, :n - rows + 21]).all() and torch.isfinite(got[0, 0, n - rows + 21:]).all()
    k, v = kv(22, 1, 1, n)
    k[0, 0, 100, 5] = float("inf")
    k[0, 0, 190, 5] = float("nan")
    cache = filled(22, k, v, 64)
    lse = torch.full((1, 2, rows), 5.0, device="cuda")
    got = call(q, lse, cache, [n], n)
    bad = torch.isnan(got[0, 0]).nonzero().flatten().tolist()
    assert bad == [100, 190]
    assert torch.isnan(call(q[:, :, :20].contiguous(), lse[:, :, :20].contiguous(), cache, [180], n)[0, 0, :180]).nonzero().flatten().tolist() == [100]


def test_memory_behind_the_last_token():
    n = 130
    k, v = kv(23, 1, 1, 192)
    k[:, :, n:] = float("nan")
    cache = filled(23, k, v, 64)
    q = normal(24, 1, 4, 2, 128).bfloat16().cuda()
    lse = torch.full((1, 4, 2), 4.0, device="cuda")
    got = call(q, lse, cache, [n], 192)
    assert torch.isfinite(got).all() and (got[0, 0, n:] == 7.0).all()


@pytest.mark.parametrize("scale", [2.0 ** -3.5, 0.01, 3.0])
def test_far_exponents(scale):
    """lse of thousands (all scores alike, and large), weights that underflow."""
    n, rows = 300, 6
    k, v = kv(25, 1, 1, n)
    k[0, 0, :, 77] = 300.0
    cache = filled(25, k, v, 64)
    q = normal(26, 1, 2, rows, 128).bfloat16().cuda()
    q[..., 77] = 30.0
    lse = attention(q, cache, [n], n, scale=scale)[1].float().cuda()
    near(call(q, lse, cache, [n], n, scale=scale), weights(q, lse, cache, [n], n, None, 1.0, rows, scale=scale), [n])


def test_after_the_calls_that_leave_lse():
    """With lse of the library's own attention a row's weights add up to one, rows of any number."""
    n = 1000
    for rows in (1, 60, 250):
        k, v = kv(27, 1, 2, n)
        cache = filled(27, k, v, 64)
        q = normal(28, 1, 8, rows, 128).bfloat16().cuda()
        lse, o = torch.empty(1, 8, rows, device="cuda"), torch.empty_like(q)
        ws = torch.empty(vs.cache_prefill_workspace(1, 8, 2, rows, n), dtype=torch.uint8, device="cuda")
        vs.cache_prefill(q, cache, o, n, lse=lse, ws=ws)
        got = call(q, lse, cache, [n], n).double().cpu()
        assert (got.sum(-1) / (4 * rows) - 1).abs().max() <= 2 * 60 * 2.0 ** -17


def test_same_bits_and_captured():
    cache, q, lse = inputs(29, 8, 2, 4, [3000, 500])
    want = call(q, lse, cache, [3000, 500], 3000)
    assert torch.equal(call(q, lse, cache, [3000, 500], 3000), want)
    lens = ints(3000, 500)
    w = torch.full((2, 2, 3000), 7.0, device="cuda")
    ws = torch.zeros(vs.cache_weigh_workspace(2, 8, 2, 4, 3000), dtype=torch.uint8, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        vs.cache_weigh(q, lse, cache, w, 3000, lens=lens, ws=ws)
    torch.cuda.synchronize()
    for now in ([3000, 500], [64, 2999], [0, 3]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        w.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, call(q, lse, cache, now, 3000))
