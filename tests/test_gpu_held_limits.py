"""The calls on held tokens at the ends of what they take: memory past 32 bits, workspaces that graphs share, streams side by side, pages of two sequences."""
import pytest
import torch

import paper_2603_04460_amd as vs
from plain_held import attention, filled, ints, kv, normal, weights

pytestmark = pytest.mark.gpu


def space(n):
    return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")


class Chain:
    """Attention of the last rows, the weights of what is held, eviction to another cache: everything that the three calls write."""

    def __init__(self, cache, q, lens, max_n, keep, ws=None):
        batch, hq, rows, _ = q.shape
        hk = cache.kv_heads
        self.cache, self.q, self.lens, self.max_n, self.keep = cache, q, ints(*lens), max_n, keep
        sizes = (vs.cache_prefill_workspace(batch, hq, hk, rows, max_n), vs.cache_weigh_workspace(batch, hq, hk, rows, max_n), vs.cache_evict_workspace(batch, hk, max_n, keep))
        self.need = max(sizes)
        self.ws = space(self.need) if ws is None else ws
        pages = -(-keep // 64)
        data = torch.full((batch * pages, hk, 1, vs.CACHE_BLOCK_BYTES), 0x5a, dtype=torch.uint8, device="cuda")
        self.to = vs.Cache(data, torch.arange(batch * pages, device="cuda").flip(0).int().view(batch, pages))
        self.o, self.lse = torch.full_like(q, 7.0), torch.full((batch, hq, rows), 7.0, device="cuda")
        self.w = torch.full((batch, hk, max_n), 7.0, device="cuda")
        self.out, self.kept = torch.full((batch, hk, keep), 7.0, device="cuda"), torch.full((batch, hk, keep), -9, dtype=torch.int32, device="cuda")
        self.after = torch.full((batch,), -9, dtype=torch.int32, device="cuda")

    def run(self, stream=None):
        vs.cache_prefill(self.q, self.cache, self.o, self.max_n, lens=self.lens, lse=self.lse, ws=self.ws, stream=stream)
        vs.cache_weigh(self.q, self.lse, self.cache, self.w, self.max_n, lens=self.lens, ws=self.ws, stream=stream)
        vs.cache_evict(self.cache, self.w, self.max_n, self.keep, self.after, lens=self.lens, n_sink=2, n_recent=9, to=self.to, weights_out=self.out, kept=self.kept,
                       ws=self.ws, stream=stream)
        return self

    def results(self):
        return [x.clone() for x in (self.o, self.lse, self.w, self.out, self.kept, self.after, self.to.data)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def chain(seed, hq, hk, rows, lens, keep, page=64, **kw):
    k, v = kv(seed, len(lens), hk, max(lens))
    return Chain(filled(seed, k, v, page), normal(seed + 3, len(lens), hq, rows, 128).bfloat16().cuda(), lens, max(lens), keep, **kw)


@pytest.mark.parametrize("rows", [1, 200])
def test_pages_past_32_bits(rows):
    near = chain(1, 8, 2, rows, [900, 333, 0], 130)
    want = near.run().results()
    have = near.cache.pages
    data = torch.empty(260000, 2, 1, vs.CACHE_BLOCK_BYTES, dtype=torch.uint8, device="cuda")
    data[-have:] = near.cache.data
    far = Chain(vs.Cache(data, near.cache.table + (260000 - have)), near.q, [900, 333, 0], 900, 130)
    assert equal(far.run().results(), want)
    # and a cache made smaller in place
    after = ints(9, 9, 9)
    for c in (near, far):
        vs.cache_evict(c.cache, c.w, 900, 130, after, lens=c.lens, n_sink=2, n_recent=9, ws=c.ws)
        assert torch.equal(after, want[5])
    assert torch.equal(data[-have:], near.cache.data)


def test_rows_past_32_bits():
    """Queries and outputs of 2^32 bytes and more: 64 heads of 300000 rows, of which 200 have a position."""
    n, rows = 200, 300000
    k, v = kv(5, 1, 1, n)
    cache = filled(5, k, v, 64)
    last = normal(8, 1, 64, n, 128).bfloat16().cuda()
    q = torch.full((1, 64, rows, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    q[:, :, -n:] = last
    o, lse = torch.full_like(q, 7.0), torch.full((1, 64, rows), 7.0, device="cuda")
    vs.cache_prefill(q, cache, o, n, lse=lse, ws=space(vs.cache_prefill_workspace(1, 64, 1, rows, n)))
    for h in range(64):
        assert (o[:, h, :-n] == 0).all()
    assert (lse[:, :, :-n] == -torch.inf).all()
    want_o, want_lse, tol_o, tol_lse = attention(last, cache, [n], n)
    assert ((o[:, :, -n:].double().cpu() - want_o).abs() <= tol_o).all() and ((lse[:, :, -n:].double().cpu() - want_lse).abs() <= tol_lse).all()
    w = torch.full((1, 1, n), 7.0, device="cuda")
    vs.cache_weigh(q, lse, cache, w, n, ws=space(vs.cache_weigh_workspace(1, 64, 1, rows, n)))
    want, tol = weights(last, lse[:, :, -n:], cache, [n], n, None, 1.0, n)
    assert ((w.double().cpu() - want).abs() <= tol).all()


def test_weights_past_32_bits():
    """1120 heads with a stride of 2^20 weights."""
    c = chain(9, 8, 8, 1, [70 - i % 3 for i in range(140)], 20)
    want = c.run().results()
    wide = torch.full((140, 8, 1 << 20), 7.0, device="cuda")
    vs.cache_weigh(c.q, c.lse, c.cache, wide, c.max_n, lens=c.lens, ws=c.ws)
    assert torch.equal(wide[:, :, :c.max_n], want[2])
    c.out.fill_(7.0), c.kept.fill_(-9), c.after.fill_(-9), c.to.data.fill_(0x5a)
    vs.cache_evict(c.cache, wide, c.max_n, c.keep, c.after, lens=c.lens, n_sink=2, n_recent=9, to=c.to, weights_out=c.out, kept=c.kept, ws=c.ws)
    assert equal(c.results()[3:], want[3:])


def test_graphs_that_share_a_workspace():
    """Of different sizes, captured one after the other, replayed in turn, with eager calls of a third in between."""
    a, b, e = chain(11, 8, 2, 300, [1500, 700], 200), chain(12, 4, 4, 140, [40000], 500), chain(13, 16, 2, 3, [900, 64, 2000], 64)
    ws = space(max(x.need for x in (a, b, e)))
    want = [x.run().results() for x in (a, b, e)]
    graphs = []
    for x in (a, b):
        x.ws = ws
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    e.ws = ws
    for turn in range(4):
        for x in (a, b, e):
            for t in (x.o, x.lse, x.w, x.out):
                t.fill_(7.0)
            x.to.data.fill_(0x5a), x.kept.fill_(-9)
        ws.random_(0, 256)
        graphs[turn % 2].replay()
        e.run()
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        for x, y in zip((a, b, e), want):
            assert equal(x.results(), y), turn


def test_streams_side_by_side():
    all_of = [chain(21, 8, 2, 250, [3000, 0, 400], 300), chain(22, 8, 2, 1, [5000, 100], 4000), chain(23, 4, 1, 40, [50000], 3000)]
    want = [x.run().results() for x in all_of]
    streams = [torch.cuda.Stream() for _ in all_of]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s in zip(all_of, streams):
            x.run(s)
    torch.cuda.synchronize()
    for x, y in zip(all_of, want):
        assert equal(x.results(), y)


@pytest.mark.parametrize("rows", [2, 150])
def test_sequences_that_share_pages(rows):
    """A prompt's pages, read for every sequence that began with it."""
    k, v = kv(31, 1, 2, 640)
    one = filled(31, k, v, 64)
    q = normal(33, 3, 4, rows, 128).bfloat16().cuda()
    shared = vs.Cache(one.data, one.table.expand(3, 10).contiguous())
    copies = vs.Cache(torch.cat([one.data] * 3), torch.cat([one.table + i * one.pages for i in range(3)]))
    lens = [640, 500, 640]
    assert equal(Chain(shared, q, lens, 640, 100).run().results(), Chain(copies, q, lens, 640, 100).run().results())
