"""The kernel for many rows of a KV head has code of its own for the running maximum, scores past 2^24, masks and V's scales: the inputs that are hard on
them, at sizes that it takes (200 and 256 rows and many blocks for each of its workgroups, seen by the workspace).  Bounds: test_gpu_cache.py."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
import plain_serving as plain
import test_gpu_cache as few

pytestmark = pytest.mark.gpu


def takes_tiles(batch, hq, hk, n_q, max_n):
    rows = hq // hk * n_q
    groups = -(-rows // 256)
    assert vs.cache_attend_workspace(batch, hq, hk, n_q, max_n) == (batch * hk + 256 // groups) * rows * 130 * 4


def test_scores_whose_rounding_exceeds_a_unit():
    takes_tiles(1, 8, 4, 100, 50000)
    few.test_attend_scores_whose_rounding_exceeds_a_unit(8, 4, 100, 50000)


@pytest.mark.parametrize("falling", [False, True])
def test_rising_maximum(falling):
    """Every block has a larger score than the ones before it, and the other way round."""
    n, hq, hk, n_q = 50000, 8, 4, 100
    takes_tiles(1, hq, hk, n_q, n)
    ramp = torch.linspace(0, 20, n).view(1, 1, n, 1)
    k = ((ramp.flip(2) if falling else ramp).expand(1, hk, n, 1) * torch.ones(128) / 8).bfloat16().cuda()
    c, q, k, v, _ = few.attend_case(401, hq, hk, n_q, [n], 256, k=k)
    q = q.abs()
    few.check(*few.call(c, q, None, n), q, k, v, [n], heads=[3])


@pytest.mark.parametrize("q_scale, scale", [(30.0, None), (1.0, 1e-4), (1.0, 3.0)])
def test_large_scores_and_scale(q_scale, scale):
    n, hq, hk, n_q = 25001, 16, 8, 128
    takes_tiles(1, hq, hk, n_q, n)
    c, q, k, v, _ = few.attend_case(402, hq, hk, n_q, [n], 64, q_scale=q_scale)
    few.check(*few.call(c, q, None, n, scale=scale), q, k, v, [n], scale=scale or 128 ** -0.5, heads=[5])


def test_scales_of_all_sizes():
    """Groups of V from 2^-120 to 2^100 beside each other and groups of zeros in every block; channels without any value."""
    n, hq, hk, n_q = 50000, 8, 4, 100
    takes_tiles(1, hq, hk, n_q, n)
    g = torch.Generator().manual_seed(403)
    x = torch.exp2(torch.randint(-120, 101, (1, hk, n, 4), generator=g).float())
    x[0, 1] = torch.exp2(torch.randint(-74, 17, (n, 4), generator=g).float())
    x[torch.rand(1, hk, n, 4, generator=g) < 0.1] = 0
    x[..., 3] = 0
    v = (torch.randn(1, hk, n, 128, generator=g) * x.repeat_interleave(32, 3)).bfloat16().cuda()
    c, q, k, _, _ = few.attend_case(404, hq, hk, n_q, [n], 192, v=v)
    o, lse = few.call(c, q, None, n)
    few.check(o, lse, q, k, v, [n], heads=[0, 1])
    assert (o[..., 96:] == 0).all()


def test_extreme_scales():
    """Values near both ends of bf16; a sequence of zeros."""
    n, hq, hk, n_q = 25000, 8, 4, 100
    takes_tiles(3, hq, hk, n_q, n)
    k, v = few.tokens(405, 3, hk, n), few.tokens(406, 3, hk, n)
    v[0] *= 2.0 ** 90
    v[1] *= 2.0 ** -110
    v[2], k[2] = 0, 0
    lens = [n, n, n]
    c, q, _, _, _ = few.attend_case(407, hq, hk, n_q, lens, 64, k=k, v=v)
    o, lse = few.call(c, q, lens, n)
    few.check(o, lse, q, k, v, lens, heads=[2])
    assert (o[2] == 0).all()


def test_rows_in_front_of_their_sequences():
    """More new tokens than a sequence holds, lengths of one and of one block, idle slots in front and behind, pages that end inside a share."""
    lens, hq, hk, n_q = [0, 1, 64, 99, 100, 101, 30000, 0, 128, 0], 4, 2, 100
    takes_tiles(10, hq, hk, n_q, 30000)
    c, q, k, v, n = few.attend_case(408, hq, hk, n_q, lens, 320)
    o, lse = few.call(c, q, lens, n)
    few.check(o, lse, q, k, v, lens, heads=[1])
    held = plain.values(*plain.quantise(few.f64(v[1, :, -1])))
    assert np.array_equal(few.f64(o[1, :, -1]), held.repeat(hq // hk, 0)) and (o[1, :, :-1] == 0).all()
