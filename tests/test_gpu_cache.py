"""The 4-bit paged cache and the attention over it against the plain form in 64 bits.

Written codes and scales, and values read back, have to be equal.  Attention: one rounding of the output to bf16 (2^-8 of it), one of
every weight (2^-8 of sum p |v|), scores off by the fp32 sum of 128 products and the exponential (2^-17 of the largest sum of |q||k| scale at
most, which moves every weight by that factor); lse by the same."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
import plain_serving as plain

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def bits16(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


def tokens(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, 128, generator=g)
    x[..., 5] *= 6.0
    x *= torch.exp2(torch.randint(-2, 3, shape + (1,), generator=g).float())
    return x.bfloat16().cuda()


def new_cache(seed, pages, kv_heads, page_size, table=None, max_pages=None):
    """Pages full of whatever was there before."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    data = torch.randint(0, 256, (pages, kv_heads, page_size // 64, vs.CACHE_BLOCK_BYTES), generator=g, dtype=torch.uint8, device="cuda")
    return vs.Cache(data, table, max_pages)


def pages_for(seed, batch, max_pages, spare=2):
    """A table of mixed-up pages and the number of pages it names them out of."""
    order = np.random.default_rng(seed).permutation(batch * max_pages + spare)[:batch * max_pages]
    return torch.from_numpy(order.reshape(batch, max_pages).astype(np.int32)).cuda(), batch * max_pages + spare


def ints(*x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def expect_blocks(before, table, page_size, k, v, lens, rows):
    """The bytes that a cache has to hold after a write: before, with the new tokens' bytes put in, as numpy."""
    data = before.cpu().numpy().copy()
    kc, ke = plain.quantise(f64(k))
    vc, ve = plain.quantise(f64(v))
    for b, n in enumerate(lens):
        for r in range(rows):
            pos = n - rows + r
            if pos < 0:
                continue
            page = table[b, pos // page_size]
            if not 0 <= page < data.shape[0]:
                continue
            for h in range(k.shape[1]):
                plain.put(data[page, h, pos % page_size // 64], pos % 64, kc[b, h, r], ke[b, h, r], vc[b, h, r], ve[b, h, r])
    return data


@pytest.mark.parametrize("page_size", [64, 192])
@pytest.mark.parametrize("rows, lens", [(1, [1, 64, 65, 0, 130]), (2, [2, 65, 1, 0, 100]), (63, [63, 100, 64, 20, 0]), (64, [64, 128, 150, 65, 3]),
                                        (131, [131, 190, 140, 0, 1])])
def test_written_bytes(rows, lens, page_size):
    """Every byte of the cache after a write: the new tokens' places hold them, all others what they held."""
    batch, hk = len(lens), 2
    max_pages = -(-192 // page_size)
    table, pages = pages_for(rows, batch, max_pages)
    c = new_cache(rows, pages, hk, page_size, table)
    k, v = tokens(1 + rows, batch, hk, rows), tokens(2 + rows, batch, hk, rows)
    want = expect_blocks(c.data, table.cpu().numpy(), page_size, k, v, lens, rows)
    vs.cache_write(c, k, v, 192, lens=ints(*lens))
    assert np.array_equal(c.data.cpu().numpy(), want)


@pytest.mark.parametrize("steps", [[1] * 70, [100, 1, 1, 30, 64, 5], [7, 13, 64, 128, 1]])
def test_written_piece_by_piece(steps):
    """A sequence written in pieces is the sequence written at once, and reads back as its plain values."""
    n, hk = sum(steps), 2
    k, v = tokens(3, hk, n), tokens(4, hk, n)
    c = new_cache(5, 8, hk, 64, max_pages=8)
    whole = vs.Cache(c.data.clone(), max_pages=8)
    vs.cache_write(whole, k, v, n)
    at = 0
    for s in steps:
        vs.cache_write(c, k[:, at:at + s].contiguous(), v[:, at:at + s].contiguous(), at + s)
        at += s
    assert torch.equal(c.data, whole.data)
    kk, vv = torch.empty_like(k), torch.empty_like(v)
    vs.cache_read(c, kk, vv, n)
    for got, x in ((kk, k), (vv, v)):
        assert np.array_equal(f64(got), plain.values(*plain.quantise(f64(x))))


def test_every_bf16_number():
    """All 65536 bit patterns, in groups of 32 of one magnitude and shuffled over all magnitudes."""
    ordered = np.arange(65536, dtype=np.uint16).reshape(2, 256, 128)
    mixed = np.random.default_rng(1).permutation(65536).astype(np.uint16).reshape(2, 256, 128)
    k, v = [torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda() for x in (ordered, mixed)]
    c = new_cache(6, 2, 2, 256, max_pages=2)
    vs.cache_write(c, k, v, 256)
    kk, vv = torch.zeros_like(k), torch.zeros_like(v)
    vs.cache_read(c, kk, vv, 256)
    for got, x in ((kk, k), (vv, v)):
        assert np.array_equal(f64(got), plain.values(*plain.quantise(f64(x))), equal_nan=True)
    c2 = new_cache(7, 2, 2, 256, max_pages=2)
    vs.cache_write(c2, v, k, 256)                        # the two sides change places
    a, b = torch.zeros_like(k), torch.zeros_like(v)
    vs.cache_read(c2, a, b, 256)
    assert np.array_equal(bits16(a), bits16(vv)) and np.array_equal(bits16(b), bits16(kk))


@pytest.mark.parametrize("rows", [1, 40, 200])
def test_read_leaves_the_rest(rows):
    """Rows in front of a sequence, idle slots and missing pages stay as they were; a range in the middle; one side alone."""
    batch, hk, page = 4, 2, 64
    lens = [200, 130, 0, 33]
    table, pages = pages_for(9, batch, 4)
    c = new_cache(8, pages, hk, page, table)
    k, v = tokens(10, batch, hk, 200), tokens(11, batch, hk, 200)
    vs.cache_write(c, k, v, 200, lens=ints(*lens))
    holed = table.clone()
    holed[0, 1], holed[1, 0], holed[3, 0] = -1, pages, 2 ** 31 - 1
    c2 = vs.Cache(c.data, holed)
    out = [torch.full((batch, hk, rows, 128), 7.5, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    vs.cache_read(c2, out[0], out[1], 200, lens=ints(*lens))
    for got, x in zip(out, (k, v)):
        want = np.full((batch, hk, rows, 128), 7.5)
        held = plain.values(*plain.quantise(f64(x)))
        for b, n in enumerate(lens):
            for r in range(rows):
                pos = n - rows + r
                if pos >= 0 and 0 <= int(holed[b, pos // page]) < pages:
                    want[b, :, r] = held[b, :, 200 - n + pos]
        assert np.array_equal(f64(got), want)
    only = torch.full_like(out[1], 7.5)
    vs.cache_read(c2, None, only, 200, lens=ints(*lens))
    assert torch.equal(only, out[1])
    only = torch.full_like(out[0], 7.5)
    vs.cache_read(c2, only, None, 200, lens=ints(*lens))
    assert torch.equal(only, out[0])
    # tokens 70 .. 99 of the first sequence
    part = torch.empty((1, hk, 30, 128), dtype=torch.bfloat16, device="cuda")
    vs.cache_read(vs.Cache(c.data, table[:1]), part, None, 100)
    assert np.array_equal(f64(part), plain.values(*plain.quantise(f64(k[:1, :, 70:100]))))


def test_write_to_missing_pages_and_past_the_bound():
    batch, hk = 3, 1
    table, pages = pages_for(12, batch, 2)
    table[0, 0], table[1, 1], table[2, 1] = -5, pages, 1 << 30
    c = new_cache(13, pages, hk, 64, table)
    k, v = tokens(14, batch, hk, 100), tokens(15, batch, hk, 100)
    lens = [100, 100, 100]
    want = expect_blocks(c.data, table.cpu().numpy(), 64, k, v, lens, 100)
    vs.cache_write(c, k, v, 100, lens=ints(2 ** 31 - 1, 100, 5000))           # lens beyond max_n count as max_n
    assert np.array_equal(c.data.cpu().numpy(), want)
    vs.cache_write(c, k, v, 128, lens=ints(-3, -2 ** 31, 0))
    assert np.array_equal(c.data.cpu().numpy(), want)


# ---- attention ----
def attend_case(seed, hq, hk, n_q, lens, page, max_n=None, table=None, q_scale=1.0, scale=None, k=None, v=None):
    """A cache with the sequences in it and a call on it: got (o, lse), wanted per sequence and head."""
    batch, longest = len(lens), max(max(lens), 1)
    max_n = longest if max_n is None else max_n
    max_pages = -(-max_n // page)
    tab, pages = pages_for(seed, batch, max_pages)
    c = new_cache(seed + 1, pages, hk, page, tab)
    k = tokens(seed + 2, batch, hk, longest) if k is None else k
    v = tokens(seed + 3, batch, hk, longest) if v is None else v
    vs.cache_write(c, k, v, max_n, lens=ints(*lens))
    g = torch.Generator().manual_seed(seed + 4)
    q = (torch.randn(batch, hq, n_q, 128, generator=g) * q_scale).bfloat16().cuda()
    return c, q, k, v, max_n


def call(c, q, lens, max_n, scale=None, ws=None):
    batch, hq, n_q, _ = q.shape
    o = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda")
    if ws is None:
        need = vs.cache_attend_workspace(batch, hq, c.kv_heads, n_q, max_n)
        ws = torch.full((max(need, 1),), 0xff, dtype=torch.uint8, device="cuda")      # NaN wherever it is read unwritten
    vs.cache_attend(q, c, o, max_n, lens=lens if isinstance(lens, torch.Tensor) or lens is None else ints(*lens), lse=lse, ws=ws, scale=scale)
    return o, lse


def check(o, lse, q, k, v, lens, scale=128 ** -0.5, heads=None, dead=None):
    """k, v [batch, hk, longest, 128]: sequence b holds the last lens[b] of them.  dead [b]: positions whose pages are missing."""
    batch, hq, n_q, _ = q.shape
    hk, longest = k.shape[1], k.shape[2]
    o, lse, q = f64(o), lse.double().cpu().numpy(), f64(q)
    for b, n in enumerate(lens):
        for h in range(hk) if heads is None else heads:
            kk, vv = [plain.values(*plain.quantise(f64(x[b, h, longest - n:]))) if n else np.zeros((0, 128)) for x in (k, v)]
            limits = n - n_q + np.arange(n_q)
            if dead is not None and len(dead[b]):
                kept = np.setdiff1d(np.arange(n), dead[b])
                kk, vv = kk[kept], vv[kept]
                limits = np.searchsorted(kept, limits, side="right") - 1
            for head in range(h * hq // hk, (h + 1) * hq // hk):
                ro, rl, size = plain.attend(q[b, head], kk, vv, limits, scale)
                off = 2.0 ** -17 * scale * (np.abs(q[b, head]).sum(1) * (np.abs(kk).max() if n and len(kk) else 0.0))
                # A weight below 2^-126 of the row's largest is below fp32's normal numbers and counts as zero: at most n such, times |v|.
                # A weight times V's scale and 2^-16 may be lost below 2^-126: times a code of at most 6 and 2^16 less than 2^-107 a key.
                lost = n * (2.0 ** -126 * (np.abs(vv).max() if len(vv) else 0.0) + 2.0 ** -107)
                bound = 2.0 ** -8 * np.abs(ro) + (2.0 ** -8 + 2 * off[:, None] + 2.0 ** -16) * size + lost
                err = np.abs(o[b, head] - ro) - bound
                assert err.max() <= 0, "sequence %d head %d row %d: %g past the bound" % (b, head, err.max(1).argmax(), err.max())
                live = np.isfinite(rl)
                assert np.array_equal(np.isneginf(lse[b, head]), ~live)
                assert (o[b, head][~live] == 0).all()
                far = np.abs(lse[b, head][live] - rl[live]) - (off[live] + 2.0 ** -21 * (1 + np.abs(rl[live])))
                assert far.max(initial=-1) <= 0, "lse of sequence %d head %d: %g past the bound" % (b, head, far.max())


@pytest.mark.parametrize("hq, hk", [(1, 1), (4, 1), (8, 2), (6, 2), (10, 2), (16, 2), (17, 1), (3, 3)])
@pytest.mark.parametrize("n_q, lens", [(1, [1, 63, 64, 65, 700]), (2, [2, 1, 66, 0, 300]), (5, [5, 3, 0, 129, 257]), (20, [20, 64, 300, 7, 1])])
def test_attend(hq, hk, n_q, lens):
    c, q, k, v, n = attend_case(hq * 100 + n_q, hq, hk, n_q, lens, 64 if hq % 2 else 128)
    check(*call(c, q, lens, n), q, k, v, lens)


@pytest.mark.parametrize("n_q, n, page", [(1, 20001, 256), (1, 40000, 1024), (3, 16400, 64), (17, 9000, 192), (128, 4111, 64), (64, 64, 64), (100, 37, 64), (33, 2049, 320)])
def test_attend_one_long_sequence(n_q, n, page):
    """Keys shared out over workgroups; chunks longer than the sequence; pages that end where blocks do and the sequence does not."""
    c, q, k, v, max_n = attend_case(n + n_q, 8, 2, n_q, [n], page)
    check(*call(c, q, None, max_n), q, k, v, [n])


@pytest.mark.parametrize("n_q, lens, max_n, hq, hk", [(100, [13001], 13001, 32, 4), (128, [30001], 60000, 8, 2), (73, [3000, 0, 40, 5001, 73], 60000, 16, 16),
                                                     (73, [3000, 0, 40, 5001, 73], 60000, 48, 16),
                                                     (128, [20000, 100, 64, 0], 20000, 33, 11)])
def test_attend_many_rows(n_q, lens, max_n, hq, hk):
    """Chunks of a hundred rows and more over long contexts: row blocks that are not full, several sequences in a share, idle ones."""
    c, q, k, v, n = attend_case(200 + n_q + hq, hq, hk, n_q, lens, 192, max_n=max_n)
    rows = hq // hk * n_q
    # the kernel for more than 160 rows: 256 rows a workgroup, its parts and one for each head
    shares = 256 // -(-rows // 256) if rows > 160 else 1024 // -(-rows // 16) // 4 * 4
    assert vs.cache_attend_workspace(len(lens), hq, hk, n_q, n) == (len(lens) * hk + shares) * rows * 130 * 4
    check(*call(c, q, lens, n), q, k, v, lens, heads=range(min(hk, 2)))


@pytest.mark.parametrize("hq, hk, n_q, n", [(1, 1, 1, 90000), (4, 1, 1, 70001), (8, 1, 2, 66000), (2, 2, 1, 131072)])
def test_attend_hundreds_of_parts(hq, hk, n_q, n):
    """One or two KV heads: every wavefront of the GPU has a block or two, hundreds of parts of a row are added up."""
    c, q, k, v, max_n = attend_case(250 + hq + n_q, hq, hk, n_q, [n], 256)
    check(*call(c, q, None, max_n), q, k, v, [n])


def test_attend_many_rows_missing_pages_and_values_that_are_not_finite():
    n, n_q, hq, hk = 50000, 100, 8, 4
    at = [n - 30, 77]
    k, v = tokens(301, 1, hk, n), tokens(302, 1, hk, n)
    v[0, 0, at[0], 40] = float("nan")
    k[0, 1, at[0], 3] = float("inf")
    c, q, _, _, _ = attend_case(300, hq, hk, n_q, [n], 256, k=k, v=v)
    o, lse = call(c, q, [n], n)
    o, lse = o.float().view(hk, hq // hk, n_q, 128), lse.view(hk, hq // hk, n_q)
    sees = torch.arange(n - n_q, n) >= at[0]
    assert torch.isnan(o[0][:, sees][..., 32:64]).all() and torch.isfinite(o[0][..., :32]).all() and torch.isfinite(o[0][..., 64:]).all()
    assert torch.isfinite(o[0][:, ~sees]).all() and torch.isfinite(lse[0]).all()
    assert torch.isnan(o[1][:, sees]).all() and torch.isnan(lse[1][:, sees]).all()
    assert torch.isfinite(o[1][:, ~sees]).all() and torch.isfinite(lse[1][:, ~sees]).all() and torch.isfinite(o[2:]).all()
    check(*call(c, q, [n], n), q, k, v, [n], heads=[2])
    table = c.table.clone()
    table[0, 3], table[0, -1], table[0, 100] = -1, c.pages, 2 ** 31 - 1
    pages = [3, table.shape[1] - 1, 100]
    dead = [np.concatenate([np.arange(256 * i, min(256 * i + 256, n)) for i in pages])]
    check(*call(vs.Cache(c.data, table), q, [n], n), q, k, v, [n], heads=[3], dead=dead)


def test_attend_bound_far_above_the_lengths():
    """Lengths far below max_n: workgroups without keys, parts that nobody writes; a full slot among idle ones."""
    lens = [5, 0, 30000, 64, 1000]
    c, q, k, v, max_n = attend_case(50, 8, 2, 1, lens, 256, max_n=100000)
    check(*call(c, q, lens, max_n), q, k, v, lens)
    lens = [0, 0, 0]
    c, q, k, v, max_n = attend_case(51, 8, 2, 4, lens, 256, max_n=100000)
    check(*call(c, q, lens, max_n), q, k, v, lens)


@pytest.mark.parametrize("batch, hq, hk, n_q", [(65, 4, 1, 1), (150, 2, 2, 1), (130, 8, 1, 3)])
@pytest.mark.parametrize("max_n", [700, 20000])
def test_attend_many_sequences(batch, hq, hk, n_q, max_n):
    """More sequences than a wavefront has lanes, of all lengths, idle ones at both ends and in the middle."""
    rng = np.random.default_rng(batch)
    lens = np.where(rng.random(batch) < 0.3, 0, np.exp(rng.uniform(0, np.log(700), batch)).astype(int))
    lens[[0, 1, 63, 64, -1]] = 0
    lens[2] = 700
    lens = [int(x) for x in lens]
    c, q, k, v, n = attend_case(100 + batch, hq, hk, n_q, lens, 64, max_n=max_n)
    check(*call(c, q, lens, n), q, k, v, lens)


def test_attend_large_scores_and_scale():
    """A softmax that one key owns, and one that is flat."""
    for q_scale, scale in ((30.0, None), (1.0, 1e-4), (1.0, 3.0)):
        lens = [300, 3000]
        c, q, k, v, n = attend_case(60, 4, 1, 3, lens, 64, q_scale=q_scale)
        check(*call(c, q, lens, n, scale=scale), q, k, v, lens, scale=scale or 128 ** -0.5)


@pytest.mark.parametrize("hq, hk, n_q, n", [(4, 1, 1, 900), (4, 1, 5, 900), (8, 2, 1, 20001), (8, 2, 5, 20001), (8, 8, 100, 30001)])
def test_attend_scores_whose_rounding_exceeds_a_unit(hq, hk, n_q, n):
    """Scores of 2^35 and more, whose last place is 2^11: one key has a score a half above all others (their sums are good to 128 roundings,
    2^-17), so it has all of the weight and the output is its value; rows of ordinary size beside them stay what they are."""
    g = torch.Generator().manual_seed(n_q)
    size = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0, 4.0])[torch.randint(0, 6, (1, hk, n), generator=g)]
    peak = n // 3
    size[:, :, peak] = 6.0
    size[:, :, n - 1] = 12.0                                # the last row's
    k = (size * 2.0 ** 13).unsqueeze(3).expand(1, hk, n, 128).bfloat16().cuda().contiguous()
    c, _, _, v, _ = attend_case(65, hq, hk, n_q, [n], 64, k=k)
    q = (2.0 ** 15 * (1 + torch.rand(1, hq, n_q, 128, generator=g))).bfloat16()
    q[:, 1::2] *= 2.0 ** -33
    q = q.cuda()
    o, lse = call(c, q, [n], n)
    for head in range(0, hq, 2):
        h = head * hk // hq
        vv = plain.values(*plain.quantise(f64(v[0, h])))
        for r in range(n_q):
            at = n - 1 if r == n_q - 1 else peak
            # (what check's `lost` allows for the other weights)
            assert (np.abs(f64(o[0, head, r]) - vv[at]) <= n * (2.0 ** -126 * np.abs(vv).max() + 2.0 ** -107)).all(), (head, r)
            want = f64(q[0, head, r]).sum() * float(k[0, h, at, 0]) * 128 ** -0.5
            assert abs(float(lse[0, head, r]) - want) <= 2.0 ** -16 * want, (head, r)
    check(o, lse, q, k, v, [n], heads=range(min(hk, 2)))     # (its bound for a large row allows anything)


def test_attend_rising_maximum():
    """Every block has a larger score than the ones before it, and the other way round."""
    n = 1500
    ramp = torch.linspace(0, 20, n).view(1, 1, n, 1)
    for k in (ramp, ramp.flip(2)):
        k = (k * torch.ones(128) / 8).bfloat16().cuda()
        lens = [n]
        c, q, k, v, n = attend_case(61, 4, 1, 1, lens, 64, k=k)
        q = q.abs()
        check(*call(c, q, lens, n), q, k, v, lens)


def test_attend_missing_pages():
    lens = [300, 200, 64, 5]
    c, q, k, v, n = attend_case(70, 8, 2, 3, lens, 64)
    table = c.table.clone()
    table[0, 1], table[0, 4], table[1, 3], table[2, :], table[3, 0] = -1, 10 ** 9, c.pages, -7, -1
    page_of = lambda b, bad: np.concatenate([np.arange(64 * i, min(64 * i + 64, lens[b])) for i in bad])
    dead = [page_of(0, [1, 4]), page_of(1, [3]), np.arange(64), np.arange(5)]
    check(*call(vs.Cache(c.data, table), q, lens, n), q, k, v, lens, dead=dead)


def test_attend_values_that_are_not_finite():
    """A NaN among a group's values makes that group's channels NaN for the rows that see the key, no others; a NaN among the keys all of
    those rows."""
    n, at = 200, 150
    k, v = tokens(80, 1, 2, n), tokens(81, 1, 2, n)
    v[0, 0, at, 40] = float("inf")
    k[0, 1, at, 3] = float("nan")
    lens = [n]
    for hq in (4, 16):                                      # two and eight heads of a KV head
        for n_q in (1, 2, 60):
            c, q, _, _, _ = attend_case(82, hq, 2, n_q, lens, 64, k=k, v=v)
            o, lse = call(c, q, lens, n)
            o, lse = o.float().view(2, hq // 2, n_q, 128), lse.view(2, hq // 2, n_q)
            sees = torch.arange(n - n_q, n) >= at
            assert torch.isnan(o[0][:, sees][..., 32:64]).all() and torch.isfinite(o[0][..., :32]).all() and torch.isfinite(o[0][..., 64:]).all()
            assert torch.isfinite(o[0][:, ~sees]).all() and torch.isfinite(lse[0]).all()
            assert torch.isnan(o[1][:, sees]).all() and torch.isnan(lse[1][:, sees]).all()
            assert torch.isfinite(o[1][:, ~sees]).all() and torch.isfinite(lse[1][:, ~sees]).all()


def test_attend_extreme_scales():
    """Values near both ends of bf16; sequences of zeros."""
    k, v = tokens(90, 3, 1, 100), tokens(91, 3, 1, 100)
    v[0] *= 2.0 ** 110
    v[1] *= 2.0 ** -110
    v[2], k[2] = 0, 0
    lens = [100, 100, 100]
    for n_q in (1, 9):
        c, q, _, _, n = attend_case(92, 4, 1, n_q, lens, 64, k=k, v=v)
        o, lse = call(c, q, lens, n)
        check(o, lse, q, k, v, lens)
        assert (o[2] == 0).all()


@pytest.mark.parametrize("n_q", [1, 5])
@pytest.mark.parametrize("n", [100, 9000])
def test_attend_scales_of_all_sizes(n_q, n):
    """Groups of V from 2^-120 to 2^100 beside each other, groups of zeros, in one block: weights whose exponents take a scale, and ones
    that cannot."""
    g = torch.Generator().manual_seed(n)
    v = torch.randn(1, 2, n, 128, generator=g)
    e = torch.randint(-120, 101, (1, 2, n, 4), generator=g)
    e[0, 1] = torch.randint(-74, 17, (n, 4), generator=g)              # at the ends of the ordinary range, and
    e[0, 1, :64] = torch.randint(-60, 10, (64, 4), generator=g)        # inside it
    x = torch.exp2(e.float())
    x[torch.rand(1, 2, n, 4, generator=g) < 0.1] = 0
    v = (v * x.repeat_interleave(32, 3)).bfloat16().cuda()
    c, q, k, _, _ = attend_case(95, 8, 2, n_q, [n], 64, v=v)[0:2] + (tokens(97, 1, 2, n), None, None)
    check(*call(c, q, [n], n), q, k, v, [n])
    padded = v.clone()
    padded[..., 64:] = 0
    c, q, _, _, _ = attend_case(95, 8, 2, n_q, [n], 64, v=padded)
    o, lse = call(c, q, [n], n)
    assert (o[..., 64:] == 0).all()
    check(o, lse, q, k, padded, [n])


def near(a, b, size):
    """Two outputs of the same sums: each is off by one rounding of itself (2^-8) and of its weights (2^-8 of sum p |v|, here `size`, itself
    an output and off by 2^-7), and scores of 128 products summed in another order move a weight by less than 2^-12."""
    a, b, size = a.float(), b.float(), size.float()
    return bool(((a - b).abs() <= 2.0 ** -8 * (a.abs() + b.abs()) + (2.0 ** -7 + 2.0 ** -11) * (1 + 2.0 ** -6) * size).all())


def test_attend_agrees_with_the_dense_call():
    """The chunk read back and attended to densely: the same sums over the same numbers, up to P's rounding in another order."""
    n, n_q, hq, hk = 1000, 100, 8, 2
    c, q, k, v, _ = attend_case(93, hq, hk, n_q, [n], 128)
    o, lse = call(c, q, [n], n)
    kk, vv = torch.empty_like(k[0]), torch.empty_like(v[0])
    vs.cache_read(c, kk, vv, n)
    o2, lse2 = torch.empty_like(q[0]), torch.empty_like(lse[0])
    vs.dense_prefill(q[0], kk, vv, o2, lse2, pos0=n - n_q)
    size = torch.empty_like(o2)
    vs.dense_prefill(q[0], kk, vv.abs(), size, None, pos0=n - n_q)
    assert float((lse[0] - lse2).abs().max()) <= 2e-3 and near(o[0], o2, size)


def test_same_call_same_bits_and_other_stream():
    lens = [5000, 70, 0, 1300]
    c, q, k, v, n = attend_case(94, 16, 4, 1, lens, 64)
    first = call(c, q, lens, n)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = call(c, q, lens, n)
    side.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32), b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


@pytest.mark.parametrize("batch, rows, hq, hk, start", [(3, 1, 8, 2, [100, 6000, 0]), (2, 4, 4, 1, [700, 64])])
def test_decoding_steps_in_a_graph(batch, rows, hq, hk, start):
    """The three calls of a decoding step, captured once with lens on the device, replayed with the eager steps between the replays:
    the same bits, and the plain form of each call on the inputs that the call before it left."""
    page, max_n = 64, 8192
    table, pages = pages_for(20, batch, max_n // page)
    freq = vs.rope_frequencies(5e5, 128, scaling=2, factor=8.0)
    rope, w = vs.Rope(freq.cuda(), 1), torch.ones(128, device="cuda")
    longest = max(start)
    k0, v0 = tokens(21, batch, hk, longest), tokens(22, batch, hk, longest)
    sets = []
    for _ in range(2):                                      # the captured and the eager program
        c = new_cache(23, pages, hk, page, table)
        vs.cache_write(c, k0, v0, max_n, lens=ints(*start))
        s = {"c": c, "lens": ints(*start), "x": torch.zeros(batch * rows, hq + 2 * hk, 128, dtype=torch.bfloat16, device="cuda"),
             "q": torch.zeros(batch, hq, rows, 128, dtype=torch.bfloat16, device="cuda"),
             "k": torch.zeros(batch, hk, rows, 128, dtype=torch.bfloat16, device="cuda"),
             "v": torch.zeros(batch, hk, rows, 128, dtype=torch.bfloat16, device="cuda"),
             "o": torch.zeros(batch, hq, rows, 128, dtype=torch.bfloat16, device="cuda"),
             "lse": torch.zeros(batch, hq, rows, device="cuda"),
             "ws": torch.empty(vs.cache_attend_workspace(batch, hq, hk, rows, max_n), dtype=torch.uint8, device="cuda")}
        sets.append(s)

    def step(s):
        x = s["x"]
        vs.qk_norm_rope(x[:, :hq], x[:, hq:hq + hk], s["q"], s["k"], rope, v=x[:, hq + hk:], v_out=s["v"], w_q=w, w_k=w, lens=s["lens"])
        vs.cache_write(s["c"], s["k"], s["v"], max_n, lens=s["lens"])
        vs.cache_attend(s["q"], s["c"], s["o"], max_n, lens=s["lens"], lse=s["lse"], ws=s["ws"])

    a, b = sets
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    keys, values = [x.clone() for x in (k0, v0)]
    lens = np.array(start)
    for i in range(6):
        x = torch.randn(batch * rows, hq + 2 * hk, 128, generator=torch.Generator().manual_seed(i)).bfloat16().cuda()
        lens = np.where(np.array(start) == 0, 0 if i < 2 else lens + rows, lens + rows)       # an idle slot that a sequence starts in
        for s in sets:
            s["x"].copy_(x)
            s["lens"].copy_(torch.from_numpy(lens.astype(np.int32)))
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        for name in ("q", "k", "v", "o", "lse"):
            assert torch.equal(a[name], b[name]), (i, name)
        assert torch.equal(a["c"].data, b["c"].data), i
        for seq in range(batch):
            if not lens[seq]:
                assert (a["o"][seq] == 0).all()
        keys, values = torch.cat([keys, a["k"]], 2), torch.cat([values, a["v"]], 2)
    for seq in range(batch):                                # a sequence's tokens are the last of its row: an idle start has added rows of its own
        n = int(lens[seq])
        check(a["o"][seq:seq + 1], a["lse"][seq:seq + 1], a["q"][seq:seq + 1], keys[seq:seq + 1], values[seq:seq + 1], [n])


def test_prompt_in_sparse_chunks_from_the_cache():
    """A prompt in chunks: norm and rotation, the chunk into the cache, all keys so far read back, sparse attention of the chunk; equal
    to one sparse call over the keys that the cache stands for.  Then a token by vs_cache_attend against the dense call."""
    hq, hk, n, chunk, page = 8, 2, 700, 256, 128
    x = tokens(30, n, hq + 2 * hk)
    rope, w = vs.Rope(vs.rope_frequencies(1e6).cuda(), 1), torch.ones(128, device="cuda")
    table, pages = pages_for(31, 1, -(-n // page))
    c = new_cache(32, pages, hk, page, table)
    from gpu_util import lists
    f = lambda a: torch.from_numpy(a).cuda()
    iv, cv = map(f, lists([np.unique(np.concatenate([[0, 1], np.random.default_rng(h).choice(n, 40)])) for h in range(hk)]))
    is_, cs = map(f, lists([np.unique(np.concatenate([np.arange(32), np.random.default_rng(9 + h).choice(n, 20)])) for h in range(hk)]))
    got, got_lse, qs = [], [], []
    for at in range(0, n, chunk):
        m = min(chunk, n - at)
        q = torch.empty(hq, m, 128, dtype=torch.bfloat16, device="cuda")
        k, v = [torch.empty(hk, m, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        part = x[at:at + m]
        vs.qk_norm_rope(part[:, :hq], part[:, hq:hq + hk], q, k, rope, v=part[:, hq + hk:], v_out=v, w_q=w, w_k=w, pos0=at)
        vs.cache_write(c, k, v, at + m)
        kk, vv = [torch.full((hk, at + m, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        vs.cache_read(c, kk, vv, at + m)
        o, lse = torch.empty_like(q), torch.empty(hq, m, device="cuda")
        ws = torch.empty(vs.sparse_prefill_workspace(hq, hk, hk, at + m), dtype=torch.uint8, device="cuda")
        vs.sparse_prefill(q, kk, vv, iv, cv, is_, cs, o, lse, ws, pos0=at)
        got.append(o)
        got_lse.append(lse)
        qs.append(q)
    q = torch.cat(qs, 1)
    o, lse = torch.empty_like(q), torch.empty(hq, n, device="cuda")
    ws = torch.empty(vs.sparse_prefill_workspace(hq, hk, hk, n), dtype=torch.uint8, device="cuda")
    vs.sparse_prefill(q, kk, vv, iv, cv, is_, cs, o, lse, ws)
    size = torch.empty_like(o)
    vs.sparse_prefill(q, kk, vv.abs(), iv, cv, is_, cs, size, None, ws)
    assert near(torch.cat(got, 1), o, size)
    assert float((torch.cat(got_lse, 1) - lse).abs().max()) <= 2e-3
    token = q[:, -1:].contiguous()
    o1, l1 = call(c, token[None], None, n)
    o2, l2 = torch.empty_like(token), torch.empty(hq, 1, device="cuda")
    vs.dense_prefill(token, kk, vv, o2, l2, pos0=n - 1)
    size = torch.empty_like(o2)
    vs.dense_prefill(token, kk, vv.abs(), size, None, pos0=n - 1)
    assert float((l1[0] - l2).abs().max()) <= 2e-3 and near(o1[0], o2, size)


def test_offsets_past_32_bits():
    """A page beyond the first 4 GiB of a cache."""
    hk, page = 2, 1024
    pages = (1 << 32) // (hk * page * 136) + 3
    data = torch.empty((pages, hk, page // 64, vs.CACHE_BLOCK_BYTES), dtype=torch.uint8, device="cuda")
    data[-2:] = 0xff
    before = data[:4].clone()
    table = ints(pages - 1, pages - 2).view(1, 2)
    c = vs.Cache(data, table)
    n = 1500
    k, v = tokens(40, 1, hk, n), tokens(41, 1, hk, n)
    vs.cache_write(c, k, v, n)
    kk, vv = torch.zeros_like(k), torch.zeros_like(v)
    vs.cache_read(c, kk, vv, n)
    assert np.array_equal(f64(kk), plain.values(*plain.quantise(f64(k)))) and np.array_equal(f64(vv), plain.values(*plain.quantise(f64(v))))
    q = tokens(42, 1, 4, 1)
    check(*call(c, q, None, n), q, k, v, [n])
    assert torch.equal(before, data[:4])


def test_refused_by_the_binding():
    c = new_cache(43, 4, 2, 64, max_pages=4)
    k = tokens(44, 1, 2, 3)
    vs.cache_write(c, k, k, 100)
    with pytest.raises(TypeError):
        vs.cache_write(c, k.float(), k, 100)
    with pytest.raises(AssertionError):
        vs.cache_write(c, k, k[:, :, :2].contiguous(), 100)
    with pytest.raises(AssertionError):
        vs.cache_write(c, tokens(45, 1, 3, 3), tokens(45, 1, 3, 3), 100)
    with pytest.raises(vs.VsError):
        vs.cache_write(c, k, k, 257)                        # more than the pages hold
    with pytest.raises(TypeError):
        vs.cache_read(c, k[:, :, ::2], None, 100)
    q = tokens(46, 1, 3, 1)
    with pytest.raises(vs.VsError):
        vs.cache_attend(q, c, torch.empty_like(q), 100)     # three heads over two
    q = tokens(46, 1, 4, 129)
    with pytest.raises(vs.VsError):
        vs.cache_attend(q, c, torch.empty_like(q), 200)
    q = tokens(47, 1, 4, 1)
    far = new_cache(48, 2, 2, 8192, max_pages=2)
    with pytest.raises(vs.VsError):
        vs.cache_attend(q, far, torch.empty_like(q), 16384)     # keys shared out: needs a workspace
    with pytest.raises(AssertionError):
        vs.Cache(c.data)
    with pytest.raises(TypeError):
        vs.Cache(c.data.cpu(), max_pages=1)
