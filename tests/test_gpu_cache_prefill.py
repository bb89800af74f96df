"""Attention of a chunk of new tokens over the 4-bit paged cache, against the plain form in 64 bits; how far it may be off is derived there."""
import pytest
import torch

import paper_2603_04460_amd as vs
from plain_held import attention, filled, held, ints, kv, normal

pytestmark = pytest.mark.gpu


def queries(seed, batch, hq, rows):
    return normal(seed, batch, hq, rows, 128).bfloat16().cuda()


def call(q, cache, lens, max_n, scale=None, fill=7.0):
    batch, hq, rows, _ = q.shape
    o = torch.full_like(q, fill)
    lse = torch.full((batch, hq, rows), fill, device="cuda")
    ws = torch.full((vs.cache_prefill_workspace(batch, hq, cache.kv_heads, rows, max_n),), 0xff, dtype=torch.uint8, device="cuda")
    vs.cache_prefill(q, cache, o, max_n, lens=None if lens is None else ints(*lens), lse=lse, ws=ws, scale=scale)
    return o, lse


def near(got, want):
    o, lse, tol_o, tol_lse = want
    for x, y, t in ((got[0], o, tol_o), (got[1], lse, tol_lse)):
        x = x.double().cpu()
        assert torch.equal(torch.isnan(x), torch.isnan(y))
        assert torch.equal(torch.isinf(x), torch.isinf(y))
        ok = torch.isfinite(y)
        worst = ((x - y).abs() - t)[ok]
        assert worst.numel() == 0 or worst.max() <= 0, (worst.max(), (x - y).abs()[ok].max())


@pytest.mark.parametrize("hq, hk", [(4, 1), (8, 1), (2, 1), (3, 1), (2, 2), (6, 3)])
@pytest.mark.parametrize("rows, lens", [(129, [129]), (200, [333, 0, 64, 200]), (257, [1, 500, 1100]), (600, [600])])
def test_heads_and_lengths(hq, hk, rows, lens):
    """Every grouping of heads; sequences shorter than the chunk, idle, of one token; the last row blocks in part."""
    batch, n = len(lens), max(lens)
    k, v = kv(rows + hq, batch, hk, n)
    cache = filled(1, k, v, 64)
    q = queries(2, batch, hq, rows)
    near(call(q, cache, lens, n), attention(q, cache, lens, n))


@pytest.mark.parametrize("page", [64, 192, 1024])
@pytest.mark.parametrize("n, rows", [(2999, 140), (4096, 320), (1111, 1111)])
def test_pages(page, n, rows):
    k, v = kv(n, 1, 2, n)
    cache = filled(3, k, v, page)
    q = queries(4, 1, 8, rows)
    near(call(q, cache, [n], n), attention(q, cache, [n], n))


def test_lengths_of_the_host():
    """No lens: every sequence holds max_n; a workspace for longer ones serves; lens outside [0, max_n] count as the nearer end."""
    k, v = kv(9, 2, 2, 700)
    cache = filled(5, k, v, 128)
    q = queries(6, 2, 4, 150)
    want = call(q, cache, [700, 700], 700)
    for lens in (None, [100000, 701]):
        for x, y in zip(call(q, cache, lens, 700), want):
            assert torch.equal(x, y)
    none = call(q, cache, [-5, 700], 700)
    assert (none[0][0] == 0).all() and torch.isinf(none[1][0]).all()
    near(none, attention(q, cache, [0, 700], 700))       # (where a row's keys are divided depends on the lengths of the batch: not the same bits)


@pytest.mark.parametrize("rows", [1, 5, 128])
def test_few_rows(rows):
    """Up to 128 rows it is vs_cache_attend, bit for bit."""
    k, v = kv(11, 2, 2, 5000)
    cache = filled(7, k, v, 64)
    q = queries(8, 2, 8, rows)
    got = call(q, cache, [5000, 777], 5000)
    o, lse = torch.empty_like(q), torch.empty(2, 8, rows, device="cuda")
    ws = torch.empty(vs.cache_attend_workspace(2, 8, 2, rows, 5000), dtype=torch.uint8, device="cuda")
    vs.cache_attend(q, cache, o, 5000, lens=ints(5000, 777), lse=lse, ws=ws)
    assert torch.equal(got[0], o) and torch.equal(got[1], lse)


@pytest.mark.parametrize("hq, hk, rows, lens, n", [(8, 2, 128, [4096] * 9 + [100, 0, 3999], 4096), (32, 4, 33, [13000, 12000], 47700), (4, 2, 65, [31000, 64], 100000)])
def test_few_rows_of_long_sequences(hq, hk, rows, lens, n):
    """Up to 128 rows where there is enough work to take this kernel: by the workspace it does."""
    batch = len(lens)
    assert vs.cache_prefill_workspace(batch, hq, hk, rows, n) > vs.cache_attend_workspace(batch, hq, hk, rows, n)
    k, v = kv(12, batch, hk, max(lens))
    cache = filled(8, k, v, 64, n=n)
    q = queries(13, batch, hq, rows)
    near(call(q, cache, lens, n), attention(q, cache, lens, n))


def test_missing_pages():
    """Tokens without a page are not attended to: in front, in the middle, behind, all of a sequence's."""
    k, v = kv(13, 4, 2, 640)
    cache = filled(9, k, v, 64)
    t = cache.table.clone()
    t[0, 0], t[0, 5], t[1, 9], t[2, :], t[3, :9] = -1, cache.pages, 2 ** 31 - 1, -7, -1
    cache.table = t
    q = queries(10, 4, 4, 300)
    lens = [640, 640, 640, 640]
    got = call(q, cache, lens, 640)
    near(got, attention(q, cache, lens, 640))
    assert (got[0][2] == 0).all() and torch.isinf(got[1][2]).all()


@pytest.mark.parametrize("spread", [3, 20, 60])
def test_values_of_all_sizes(spread):
    """V whose scales lie far apart, rising, falling and mixed; groups of zeros among them."""
    n, rows = 900, 200
    k, v = kv(15, 3, 1, n)
    exps = torch.randint(-spread, spread + 1, (3, 1, n, 4), generator=torch.Generator().manual_seed(16))
    exps[0] = exps[0].sort(dim=1).values
    exps[1] = exps[1].sort(dim=1, descending=True).values
    x = v.float().cpu().unflatten(-1, (4, 32)) * torch.exp2(exps.float()).unsqueeze(-1)
    x[2, :, 100:120, 1] = 0.0
    v = x.flatten(-2).bfloat16().cuda()
    cache = filled(11, k, v, 64)
    q = queries(12, 3, 4, rows)
    near(call(q, cache, [n] * 3, n), attention(q, cache, [n] * 3, n))


@pytest.mark.parametrize("big", [2.0 ** 15, 2.0 ** 40, 1e25])
def test_large_values_that_some_rows_do_not_see(big):
    """A value of a late token must not take precision from the rows in front of it, nor one that nobody looks at from the others."""
    n, rows = 512, 256
    k, v = kv(17, 2, 1, n)
    v[0, :, 450] *= big
    v[1, :, 3] *= big
    k[1, :, 3] = 0.0
    k[1, :, 3, 9] = -200.0
    q = queries(14, 2, 4, rows)
    q[1, :, :, 9] = 200.0                                # scores of -3500: a weight of zero
    cache = filled(13, k, v, 64)
    near(call(q, cache, [n, n], n), attention(q, cache, [n, n], n))


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_values_that_are_not_finite(what):
    """They reach the rows that see them, in their 32 channels, and no other."""
    n, rows = 400, 260
    k, v = kv(19, 2, 2, n)
    v[0, 1, 300, 40] = what
    v[1, 0, 399, 127] = what
    cache = filled(15, k, v, 64)
    q = queries(16, 2, 4, rows)
    got, want = call(q, cache, [n, n], n), attention(q, cache, [n, n], n)
    near(got, want)
    assert torch.isnan(got[0][0, 2:, 160:, 32:64]).all() and torch.isnan(got[0]).sum() == 2 * 100 * 32 + 2 * 1 * 32


def test_keys_that_are_not_finite():
    """A key that is not finite reaches the rows that see it; behind the last token anything may stand."""
    n, rows = 300, 200
    k, v = kv(21, 2, 1, n)
    k[0, 0, 250, 3] = float("nan")
    cache = filled(17, k, v, 64)
    q = queries(18, 2, 4, rows)
    o, lse = call(q, cache, [n, 170], n)
    assert torch.isnan(o[0, :, 150:]).all() and torch.isnan(lse[0, :, 150:]).all()
    near((o[:1, :, :150], lse[:1, :, :150]), attention(q[:1, :, :150], filled(17, k[:1, :, :250].contiguous(), v[:1, :, :250].contiguous(), 64), [250], 250))
    near((o[1:], lse[1:]), tuple(x[1:] for x in attention(q, cache, [0, 170], n)))


def test_memory_behind_the_last_token():
    """Pages are not cleared: every byte behind the last token set to what is worst."""
    n, rows = 330, 150
    k, v = kv(23, 1, 2, n)
    cache = filled(19, k, v, 64)
    q = queries(20, 1, 4, rows)
    want = call(q, cache, [n], n)
    k3, v3 = kv(24, 1, 2, 384)
    k3[:, :, :n], v3[:, :, :n] = k, v
    k3[:, :, n:] = float("nan")
    v3[:, :, n:] = float("inf")
    for x, y in zip(call(q, filled(19, k3, v3, 64), [n], n), want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("way", ["rising", "falling", "steps"])
@pytest.mark.parametrize("factor", [1.0, 30.0])
def test_running_maximum(way, factor):
    """Scores that grow and fall over the sequence, in every row or in single ones."""
    n, rows = 1500, 160
    k, v = kv(25, 1, 1, n)
    t = torch.linspace(0, 1, n)
    t = {"rising": t, "falling": 1 - t, "steps": (t * 6).floor() / 6}[way]
    k[0, 0] = (torch.randn(n, 128, generator=torch.Generator().manual_seed(1)) * 0.1).bfloat16().cuda()
    k[0, 0, :, 9] = (t * 20 * factor).bfloat16().cuda()
    q = queries(22, 1, 4, rows)
    q[..., 9] = 8.0
    q[:, 1, ::3, 9] = -8.0
    cache = filled(21, k, v, 64)
    near(call(q, cache, [n], n), attention(q, cache, [n], n))


def test_large_scores():
    """Scores past 2^24: their rounding is a unit and more, the row's largest weight is one all the same."""
    n, rows = 256, 150
    k, v = kv(27, 1, 1, n)
    k[0, 0] = 0.0
    k[0, 0, :, 0] = torch.exp2(torch.arange(n) % 16 - 8.0).bfloat16().cuda()
    q = torch.zeros(1, 1, rows, 128, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 26
    cache = filled(23, k, v, 64)
    o, lse = call(q, cache, [n], n, scale=1.0)
    kk, vv = held(cache, n, 1)
    for r in range(rows):
        seen = n - rows + r + 1
        s = kk[0, 0, :seen, 0]
        at = s == s.max()
        want = vv[0, 0, :seen][at].mean(0)
        mass = vv[0, 0, :seen][at].abs().mean(0)
        assert ((o[0, 0, r].double().cpu() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -10 * mass).all()
        assert abs(lse[0, 0, r].item() / (s.max().item() * 2.0 ** 26) - 1) <= 2.0 ** -21


def test_many_sequences():
    """More sequences than a wavefront has lanes, most of them short."""
    lens = [(37 * i) % 150 for i in range(70)]
    k, v = kv(33, 70, 1, 150)
    cache = filled(29, k, v, 64)
    q = queries(28, 70, 2, 131)
    near(call(q, cache, lens, 150), attention(q, cache, lens, 150))


@pytest.mark.parametrize("hq, hk, rows, n", [(1, 1, 267, 9000), (4, 1, 130, 20000), (3, 3, 400, 5000)])
def test_many_parts(hq, hk, rows, n):
    """Few units of many keys: dozens of workgroups share each; a row that is not a number stays alone."""
    k, v = kv(41, 1, hk, n)
    cache = filled(41, k, v, 64)
    cache.table[0, 3:40] = -1
    q = queries(42, 1, hq, rows)
    q[0, 0, 77] = float("nan")
    near(call(q, cache, [n], n), attention(q, cache, [n], n))


def test_stream():
    """On a stream of its own, beside another call with another workspace."""
    k, v = kv(35, 1, 2, 2000)
    cache = filled(31, k, v, 64)
    qs = [queries(30 + i, 1, 8, 200 + 50 * i) for i in range(2)]
    want = [call(q, cache, [2000], 2000) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    got = [(torch.zeros_like(q), torch.zeros(1, 8, q.shape[2], device="cuda"), torch.zeros(vs.cache_prefill_workspace(1, 8, 2, q.shape[2], 2000), dtype=torch.uint8, device="cuda"))
           for q in qs]
    torch.cuda.synchronize()
    for _ in range(3):
        for q, (o, lse, ws), s in zip(qs, got, streams):
            vs.cache_prefill(q, cache, o, 2000, lse=lse, ws=ws, stream=s)
    torch.cuda.synchronize()
    for (o, lse, _), w in zip(got, want):
        assert torch.equal(o, w[0]) and torch.equal(lse, w[1])


def test_queries_that_are_not_finite():
    """A row whose query is not finite is not a number; the other rows of its tile are what they are."""
    k, v = kv(37, 1, 1, 500)
    cache = filled(33, k, v, 64)
    q = queries(34, 1, 4, 180)
    q[0, 2, 77, 5], q[0, 1, 0, 0] = float("nan"), float("nan")
    got = call(q, cache, [500], 500)
    assert torch.isnan(got[0][0, 2, 77]).all() and torch.isnan(got[1][0, 1, 0])
    near(got, attention(q, cache, [500], 500))


def test_same_bits():
    k, v = kv(29, 3, 2, 3000)
    cache = filled(25, k, v, 64)
    q = queries(24, 3, 8, 333)
    first = call(q, cache, [3000, 1234, 400], 3000)
    for fill in (0.0, float("nan")):
        for x, y in zip(call(q, cache, [3000, 1234, 400], 3000, fill=fill), first):
            assert torch.equal(x, y)


def test_captured():
    """A captured call, replayed for other lengths and other tokens in the same memory, with eager work between."""
    k, v = kv(31, 2, 2, 1500)
    cache = filled(27, k, v, 64)
    q, lens = queries(26, 2, 8, 200), ints(1500, 700)
    o, lse = torch.zeros_like(q), torch.zeros(2, 8, 200, device="cuda")
    ws = torch.zeros(vs.cache_prefill_workspace(2, 8, 2, 200, 1500), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        vs.cache_prefill(q, cache, o, 1500, lens=lens, lse=lse, ws=ws)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            vs.cache_prefill(q, cache, o, 1500, lens=lens, lse=lse, ws=ws)
    torch.cuda.synchronize()
    for step, now in enumerate(([1500, 700], [201, 1500], [0, 90], [1500, 1499])):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        q.copy_(queries(40 + step, 2, 8, 200))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((o, lse), call(q, cache, now, 1500)):
            assert torch.equal(x, y), now
