"""vs_qk_norm_rope against the plain form in 64 bits.

Tolerance: one rounding to bf16 (2^-8 of the value) and the fp32 arithmetic in front of it, which is relative to the rotated pair:
the angle is off by 2^-24 of a turn at most (2 pi 2^-25 and the sine's own 2^-23), the norm by 2^-20 (a sum of 128 squares, a root, two
products); 2^-18 of |a| + |b| covers both."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
import plain_serving as plain

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def packed(seed, tokens, heads, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(tokens, heads, 128, generator=g) * (0.5 + torch.rand(heads, 128, generator=g)) * scale).bfloat16().cuda()


def weight(seed):
    g = torch.Generator().manual_seed(seed + 77)
    return (1.0 + 0.2 * torch.randn(128, generator=g)).float().cuda()


def heads_first(x, batch, rows):
    return f64(x).reshape(batch, rows, x.shape[1], 128).transpose(0, 2, 1, 3)


def check(got, x, w, eps, freq, positions, pairing, magnitude=1.0):
    """got [batch, heads, rows, 128], x the same in 64 bits, positions [batch, rows]"""
    got, wt = f64(got), None if w is None else f64(w)
    for b in range(x.shape[0]):
        ref = plain.norm_rope(x[b], wt, eps, freq, positions[b], pairing, magnitude)
        pair = np.abs(plain.norm_rope(x[b], wt, eps, 0 * freq, positions[b], pairing, magnitude))
        i = np.arange(len(freq))
        i, j = (2 * i, 2 * i + 1) if pairing == 0 else (i, i + len(freq))
        pair[..., i] = pair[..., j] = pair[..., i] + pair[..., j]
        assert np.isfinite(got[b]).all()
        bad = np.abs(got[b] - ref) - (2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * pair)
        assert bad.max() <= 0, "%g past the bound, sequence %d" % (bad.max(), b)


@pytest.mark.parametrize("rot", [8, 64, 72, 96, 128])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("batch, rows, hq, hk", [(1, 1, 1, 1), (1, 33, 4, 1), (5, 3, 8, 2), (19, 1, 32, 8), (1, 700, 5, 5)])
def test_against_the_formula(batch, rows, hq, hk, pairing, rot):
    x = packed(rows * 31 + rot, batch * rows, hq + 2 * hk)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    freq = vs.rope_frequencies(5e5, rot, scaling=2, factor=8.0)
    rope = vs.Rope(freq.cuda(), pairing)
    w_q, w_k = weight(1), weight(2)
    rng = np.random.default_rng(batch)
    lens = rng.integers(rows, 1 << 20, batch)
    lens[0] = 1 << 20
    if batch > 3:
        lens[1], lens[2] = 1, 0                          # rows in front of the sequence
    out = [torch.full((batch, h, rows, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk)]
    vs.qk_norm_rope(q, k, out[0], out[1], rope, v=v, v_out=out[2], w_q=w_q, w_k=w_k, eps=1e-5, lens=torch.tensor(lens, dtype=torch.int32).cuda())
    pos = lens[:, None] - rows + np.arange(rows)
    check(out[0], heads_first(q, batch, rows), w_q, 1e-5, freq.numpy(), pos, pairing)
    check(out[1], heads_first(k, batch, rows), w_k, 1e-5, freq.numpy(), pos, pairing)
    assert np.array_equal(f64(out[2]), heads_first(v, batch, rows))


@pytest.mark.parametrize("rows", [1, 5, 130, 4097])
@pytest.mark.parametrize("which", ["neither", "q", "k"])
def test_without_norm_values_or_lens(rows, which):
    """A norm for one of the two, no values, positions from pos0, a magnitude, heads first on the input side."""
    hq, hk, pos0 = 4, 2, 130000
    g = torch.Generator().manual_seed(rows)
    q, k = [torch.randn(h, rows, 128, generator=g).bfloat16().cuda() for h in (hq, hk)]
    w = weight(3)
    w_q, w_k = w if which == "q" else None, w if which == "k" else None
    freq = vs.rope_frequencies(1e6, 64, scaling=1, factor=4.0)
    out = [torch.full_like(t, float("nan")) for t in (q, k)]
    vs.qk_norm_rope(q.transpose(0, 1), k.transpose(0, 1), out[0], out[1], vs.Rope(freq.cuda(), 1, magnitude=1.25), w_q=w_q, w_k=w_k, pos0=pos0)
    pos = (pos0 + np.arange(rows))[None]
    for got, x, wt in ((out[0], q, w_q), (out[1], k, w_k)):
        check(got[None], f64(x)[None], wt, 1e-6, freq.numpy(), pos, 1, 1.25)
    inplace = [q.clone(), k.clone()]
    vs.qk_norm_rope(inplace[0].transpose(0, 1), inplace[1].transpose(0, 1), inplace[0], inplace[1], vs.Rope(freq.cuda(), 1, magnitude=1.25),
                    w_q=w_q, w_k=w_k, pos0=pos0)
    assert all(torch.equal(a, b) for a, b in zip(inplace, out))


def test_agrees_with_rope_apply():
    """Without norm and scaling it is vs_rope_apply: the same bf16 numbers but for pairs next to a rounding border."""
    q = packed(8, 1000, 3)
    for pairing in (0, 1):
        want = q.transpose(0, 1).contiguous()
        out = [torch.empty_like(want), torch.empty_like(want)]
        vs.qk_norm_rope(q, q, out[0], out[1], vs.Rope(vs.rope_frequencies(1e6).cuda(), pairing), pos0=120000)
        vs.rope_apply(want, 120000, 1e6, pairing)
        assert torch.equal(out[0], out[1])
        far = (out[0].view(torch.int16).int() - want.view(torch.int16).int()).abs()
        assert float((far != 0).float().mean()) < 2.0 ** -10 and float((out[0].float() - want.float()).abs().max()) <= 2.0 ** -6


def test_strides_of_a_wider_projection():
    """Parts of a projection that holds more than q, k and v, and heads that are not next to each other."""
    wide = packed(4, 50, 20)
    q, k, v = wide[:, 1:9:2], wide[:, 10:12], wide[:, 15:17]
    freq = vs.rope_frequencies(1e6)
    rope = vs.Rope(freq.cuda(), 1)
    w = weight(4)
    out = [torch.empty((1, h, 50, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
    vs.qk_norm_rope(q, k, out[0], out[1], rope, v=v, v_out=out[2], w_q=w, w_k=w, pos0=7)
    pos = 7 + np.arange(50)[None]
    check(out[0], heads_first(q, 1, 50), w, 1e-6, freq.numpy(), pos, 1)
    check(out[1], heads_first(k, 1, 50), w, 1e-6, freq.numpy(), pos, 1)
    assert torch.equal(out[2][0], v.transpose(0, 1))


def test_extreme_rows():
    """Rows of zeros, of the largest and of the smallest numbers, with a NaN, with an infinity."""
    x = packed(6, 6, 1)
    x[1] = 0
    x[2] = x[2].sign() * 3e38
    x[3] *= 1e-30
    x[4, 0, 17] = float("nan")
    x[5, 0, 3] = float("inf")
    w = weight(5)
    freq = vs.rope_frequencies(1e6)
    out = [torch.empty((1, 1, 6, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    vs.qk_norm_rope(x, x, out[0], out[1], vs.Rope(freq.cuda(), 1), w_q=w, w_k=w)
    check(out[0][:, :, :4], heads_first(x, 1, 6)[:, :, :4], w, 1e-6, freq.numpy(), np.arange(4)[None], 1)
    assert (out[0][0, 0, 1] == 0).all() and torch.isnan(out[0][0, 0, 4]).all()
    row = f64(out[0])[0, 0, 5]
    assert np.isnan(row[[3, 67]]).all() and (np.delete(row, [3, 67]) == 0).all()


def test_refused_by_the_binding():
    x = packed(1, 4, 3)
    out = torch.empty((1, 1, 4, 128), dtype=torch.bfloat16, device="cuda")
    rope = vs.Rope(vs.rope_frequencies(1e6).cuda())
    a, b = x[:, :1], x[:, 1:2]
    vs.qk_norm_rope(a, b, out, out.clone(), rope)
    with pytest.raises(TypeError):
        vs.qk_norm_rope(a.float(), b, out, out.clone(), rope)
    with pytest.raises(TypeError):
        vs.qk_norm_rope(a, b, out.float(), out.clone(), rope)
    with pytest.raises(TypeError):
        vs.Rope(vs.rope_frequencies(1e6))
    with pytest.raises(AssertionError):
        vs.qk_norm_rope(a[:3], b, out, out.clone(), rope)
    with pytest.raises(AssertionError):
        vs.qk_norm_rope(a, b, out, out.clone(), rope, v=b)
    with pytest.raises(TypeError):
        vs.qk_norm_rope(a, b, out, out.clone(), rope, lens=torch.zeros(1, dtype=torch.int64, device="cuda"))
