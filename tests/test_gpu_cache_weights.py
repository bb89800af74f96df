"""How exactly vs_cache_attend holds its weights: sums of V that cancel to a three-hundredth of their parts.

Two kinds of keys, shuffled: A (K = 6 in the row's only channel, V = 1) and B (K = 4, V = -2, -4, -8, -16 in the four groups of channels), and a
row q = t, so that with w = exp(-2 t scale) and nA, nB keys in sight
    o = (nA - nB 2^(g+1) w) / (nA + nB w),      size = (nA + nB 2^(g+1) w) / (nA + nB w).
scale makes w = (1 + 2^-8) / 2 for t = 1: halfway between two bf16 numbers, 2^-8 off both.
Bound: the output's rounding (2^-8 |o|); a weight in two bf16 terms (the first cut off, 2^-7, the second rounded, 2^-8 of it): 2^-15; exponents of
at most 16 in fp32 (product, sum and factor rounded, 3 * 2^-24 * 16, times ln 2) and the exponential (2^-22): below 2^-18, in the weights and in
their sum; fp32 sums in chains of at most 2048 additions (blocks of a worker x 64 keys x two terms): 2^-13.  In all 2^-8 |o| + 2^-12 size; with
weights of one bf16 term a row is off by 2^-9 size and more."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs

pytestmark = pytest.mark.gpu

SCALE = float(np.float32(-np.log((1 + 2.0 ** -8) / 2) / 2))


# the forms: a workgroup for each head and the row of all blocks, each with 4 and with 16 rows a tile; 256 rows a workgroup
@pytest.mark.parametrize("hq, hk, n_q, n, form", [(4, 1, 1, 900, "head"), (8, 2, 3, 1000, "head"), (8, 1, 20, 700, "head"),
                                                  (4, 1, 1, 40001, "row"), (8, 2, 1, 20001, "row"), (8, 2, 5, 20001, "row"), (16, 4, 30, 9000, "row"),
                                                  (8, 4, 100, 50000, "tile"), (16, 8, 128, 25001, "tile")])
def test_weights_of_two_terms(hq, hk, n_q, n, form):
    rows, need = hq // hk * n_q, vs.cache_attend_workspace(1, hq, hk, n_q, n)
    shares = {"head": 0, "row": 1024 // -(-rows // (4 if rows <= 4 else 16)) // 4 * 4, "tile": 256 // -(-rows // 256)}[form]
    assert need == (shares and (hk + shares) * rows * 130 * 4)
    g = torch.Generator().manual_seed(n)
    is_b = torch.rand(hk, n, generator=g) < 0.5
    is_b[:, 0], is_b[:, 1] = False, True
    k = torch.where(is_b, 4.0, 6.0).unsqueeze(2).repeat(1, 1, 128)
    v = torch.where(is_b.unsqueeze(2), -torch.exp2(torch.arange(4).repeat_interleave(32) + 1.0), 1.0)
    c = vs.Cache(torch.zeros(-(-n // 256), hk, 4, vs.CACHE_BLOCK_BYTES, dtype=torch.uint8, device="cuda"), max_pages=-(-n // 256))
    vs.cache_write(c, k.bfloat16().cuda(), v.bfloat16().cuda(), n)
    q, t = torch.zeros(1, hq, n_q, 128), torch.ones(hq, n_q)
    t[:, 1::3], t[:, 2::3] = 2.0, 0.5
    at = 37 * torch.arange(hq) % 128
    q[0, torch.arange(hq), :, at] = t
    q, t = q.bfloat16().cuda(), t.double().numpy()
    o, ws = torch.full_like(q, float("nan")), torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    vs.cache_attend(q, c, o, n, ws=ws, scale=SCALE)
    o, last = o[0].double().cpu().numpy(), n - n_q + np.arange(n_q)
    for head in range(hq):
        b = np.cumsum(is_b[head * hk // hq].numpy())[last].astype(np.float64)[:, None]
        a, w = last[:, None] + 1 - b, np.exp(-2 * t[head] * SCALE)[:, None]
        part = b * w * np.exp2(np.arange(4) + 1.0).repeat(32)
        want, size = (a - part) / (a + b * w), (a + part) / (a + b * w)
        bad = np.abs(o[head] - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -12 * size)
        assert bad.max() <= 0, "head %d row %d: %g past the bound" % (head, bad.max(1).argmax(), bad.max())
