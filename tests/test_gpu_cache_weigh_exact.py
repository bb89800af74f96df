"""Weights of held tokens where every product is exact, so that the only errors are those of scale log2(e), of lse's share of the exponent and of the exponential:
the exponents' own precision, at lse of any size."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
from plain_held import filled

pytestmark = pytest.mark.gpu

FORMS = [(2, 6, 1), (2, 40, 1), (4, 300, 2)]               # query heads, rows, KV heads: 12 rows in registers; tiles that stay in LDS; that do not


def call(q, lse, cache, n, scale, decay=1.0):
    batch, hq, rows, _ = q.shape
    out = torch.full((batch, cache.kv_heads, n), 7.0, device="cuda")
    ws = torch.full((vs.cache_weigh_workspace(batch, hq, cache.kv_heads, rows, n),), 0xff, dtype=torch.uint8, device="cuda")
    vs.cache_weigh(q, lse, cache, out, n, ws=ws, scale=scale)
    return out.double().cpu().numpy()[0]


def check(s, lse, got, scale, rows):
    """s [heads, rows, n] exact scores, lse [heads, rows] as given.  The kernel's exponent is (c / scale)(scale s - lse) with c = scale log2(e) in fp32 (two roundings,
    2^-23), rounded as a difference (2^-24 of itself); c / scale in two terms, for lse up to 2^22, is off by less than 2^-47; exponentials and their factor by 2^-22; then
    the fp32 sums."""
    heads, _, n = s.shape
    scale = float(np.float32(scale))
    seen = np.arange(n) <= (n - rows + np.arange(rows))[:, None]
    l = lse.double().cpu().numpy()[0][..., None]
    t = scale * s - l
    with np.errstate(over="ignore"):
        p = np.where(seen, np.exp(np.minimum(t, 700.0)), 0.0)
        relative = np.abs(t) * 2.0 ** -22 + np.minimum(np.abs(l), 2.0 ** 22) * 2.0 ** -46 + 2.0 ** -21
        tol = (p * relative).sum((0, 1)) + (heads * rows + 2) * 2.0 ** -24 * p.sum((0, 1)) + heads * rows * 2.0 ** -126
    want = p.sum((0, 1))
    assert not np.isnan(got).any()
    over = want > 2.0 ** 127
    assert np.isinf(got[want > 2.0 ** 129]).all()
    worst = np.abs(got - want)[~over] / tol[~over]
    assert worst.size == 0 or worst.max() <= 1, (worst.max(), np.abs(got / np.maximum(want, 1e-300) - 1)[~over].max())


@pytest.mark.parametrize("hq, rows, hk", FORMS)
@pytest.mark.parametrize("scale", [2.0 ** -3.5, 0.01, 1.0, 3.0])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 13, 2.0 ** 15])
def test_exponents_near_zero_of_large_terms(hq, rows, hk, scale, size):
    """All scores near size / scale, lse beside them: what counts is their difference."""
    n, group = 700, hq // hk
    g = torch.Generator().manual_seed(71)
    large = 2.0 ** round(np.log2(size / scale))
    step = 2.0 ** round(np.log2(1.0 / scale))              # of a score, one unit of the exponent
    k = torch.zeros(1, hk, n, 128)
    k[..., 0] = 2.0 ** 6
    k[..., 32] = torch.tensor([-6.0, -4.0, -3.0, -2.0, -1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5, 2.0])[torch.randint(0, 12, (1, hk, n), generator=g)]
    cache = filled(71, k.bfloat16().cuda(), k.bfloat16().cuda(), 64)
    q = torch.zeros(1, hq, rows, 128)
    q[..., 0] = large / 2.0 ** 6
    q[..., 32] = step * torch.randint(1, 4, (1, hq, rows), generator=g)
    lse = (float(np.float32(scale)) * large + 6.0 * torch.rand(1, hq, rows, generator=g, dtype=torch.float64)).float().cuda()
    got = call(q.bfloat16().cuda(), lse, cache, n, scale)
    s = (q[0].double() @ k[0].double().repeat_interleave(group, 0).transpose(-1, -2)).numpy()
    for h in range(hk):
        heads = slice(h * group, (h + 1) * group)
        check(s[heads], lse[:, heads], got[h], scale, rows)


@pytest.mark.parametrize("hq, rows, hk", FORMS)
@pytest.mark.parametrize("scale", [0.1, 0.75, 1.0])
@pytest.mark.parametrize("exponent", [20, 26, 29, 30, 31, 32, 33, 36, 60])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_lse_of_any_size(hq, rows, hk, scale, exponent, sign):
    """lse whose own steps are units and more: keys that the row does not see, and those far below, have a weight of zero whatever the others have."""
    n, group = 500, hq // hk
    g = torch.Generator().manual_seed(73)
    k = torch.zeros(1, hk, n, 128)
    k[..., 7] = torch.tensor([1.0, 1.0, 1.5, 2.0])[torch.randint(0, 4, (1, hk, n), generator=g)]
    cache = filled(73, k.bfloat16().cuda(), k.bfloat16().cuda(), 64)
    q = torch.zeros(1, hq, rows, 128)
    q[..., 7] = sign * torch.randint(128, 256, (1, hq, rows), generator=g) * 2.0 ** (exponent - 7)
    # the row's largest score, as an attention leaves it: in fp32
    lse = (q[..., 7].double() * (2.0 if sign > 0 else 1.0) * float(np.float32(scale))).float().cuda()
    got = call(q.bfloat16().cuda(), lse, cache, n, scale)
    s = (q[0].double() @ k[0].double().repeat_interleave(group, 0).transpose(-1, -2)).numpy()
    for h in range(hk):
        heads = slice(h * group, (h + 1) * group)
        check(s[heads], lse[:, heads], got[h], scale, rows)


@pytest.mark.parametrize("rows", [10, 150])
def test_after_the_attention_of_large_scores(rows):
    """lse of 2^33 as vs_cache_prefill leaves it: no weight is NaN, those of keys that are far below are zero."""
    n = 256
    k = torch.zeros(1, 1, n, 128)
    k[0, 0, :, 0] = torch.exp2(torch.arange(n) % 16 - 8.0)
    cache = filled(75, k.bfloat16().cuda(), k.bfloat16().cuda(), 64)
    q = torch.zeros(1, 2, rows, 128, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 26 * (1 + torch.arange(rows, device="cuda") % 64 / 64)
    o, lse = torch.empty_like(q), torch.empty(1, 2, rows, device="cuda")
    ws = torch.empty(vs.cache_prefill_workspace(1, 2, 1, rows, n), dtype=torch.uint8, device="cuda")
    vs.cache_prefill(q, cache, o, n, lse=lse, ws=ws, scale=1.0)
    got = call(q, lse, cache, n, 1.0)[0]
    assert not np.isnan(got).any()
    assert (got[np.arange(n) % 16 != 15] == 0).all()
