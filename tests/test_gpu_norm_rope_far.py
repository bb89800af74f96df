"""vs_qk_norm_rope at the end of its positions.

Tolerance: the output's rounding, 2^-8 of it, and 2^-19 of |a| + |b|, the rotated pair: the fraction of a turn is reduced in fp64 (three roundings, 3 * 2^-53 of an
angle of 2^31: 2^-20.4) and rounded to fp32 (at most half a turn: 2 pi 2^-26); sine and cosine 2^-23; norm, weight, magnitude and the two products
fewer than 13 roundings of 2^-24: in all below 2^-20.1 + 2^-20.4."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
import test_gpu_norm_rope as norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pos0, rows", [(0, 64), ((1 << 20) - 500, 1000), ((1 << 24) - 7, 2000), ((1 << 31) - 1000, 1000)])
@pytest.mark.parametrize("pairing", [0, 1])
def test_far_positions(pos0, rows, pairing):
    """Angles in 80 bits here: in 64 the product alone is 2^-22 off at 2^31."""
    hq, hk = 6, 1
    x = norm.packed(rows, rows, hq + hk)
    freq = vs.rope_frequencies(5e5, 128, scaling=2, factor=8.0)
    w = norm.weight(7)
    out = [torch.empty(h, rows, 128, dtype=torch.bfloat16, device="cuda") for h in (hq, hk)]
    vs.qk_norm_rope(x[:, :hq], x[:, hq:], out[0], out[1], vs.Rope(freq.cuda(), pairing), w_q=w, w_k=w, pos0=pos0)
    t = (pos0 + np.arange(rows)).astype(np.longdouble)[:, None] * freq.numpy().astype(np.longdouble)
    c, s = np.cos(t).astype(np.float64), np.sin(t).astype(np.float64)
    p = np.arange(64)
    i, j = (2 * p, 2 * p + 1) if pairing == 0 else (p, p + 64)
    y = norm.heads_first(x, 1, rows)[0]
    y = y / np.sqrt((y * y).mean(-1, keepdims=True) + 1e-6) * norm.f64(w)
    a, b = y[..., i], y[..., j]
    got = np.concatenate([norm.f64(o) for o in out])
    for at, want in ((i, a * c - b * s), (j, a * s + b * c)):
        bad = np.abs(got[..., at] - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -19 * (np.abs(a) + np.abs(b)))
        assert bad.max() <= 0, "%g past the bound" % bad.max()
