"""A cache that grows between calls: more pages for a sequence by a wider table, then all pages in a larger array."""
import pytest
import torch

import paper_2603_04460_amd as vs
import test_gpu_cache as few

pytestmark = pytest.mark.gpu


def test_growing_cache():
    hq, hk, page, n = 4, 1, 64, 500
    k, v = few.tokens(501, 1, hk, n), few.tokens(502, 1, hk, n)
    c = few.new_cache(503, 4, hk, page, few.ints(2, 0, 3).view(1, 3))
    vs.cache_write(c, k[:, :, :150].contiguous(), v[:, :, :150].contiguous(), 150)
    with pytest.raises(vs.VsError):                         # 500 tokens do not fit in three pages
        vs.cache_write(c, k[:, :, 150:].contiguous(), v[:, :, 150:].contiguous(), n)
    c.table = few.ints(2, 0, 3, 5, 9, 8, 1, 4).view(1, 8)
    grown = few.new_cache(504, 10, hk, page, max_pages=1).data
    grown[:4] = c.data
    c.data = grown
    vs.cache_write(c, k[:, :, 150:].contiguous(), v[:, :, 150:].contiguous(), n)
    q = few.tokens(505, 1, hq, 2)
    few.check(*few.call(c, q, None, n), q, k, v, [n])
    rope = vs.Rope(vs.rope_frequencies(1e6).cuda(), 1)
    x = few.tokens(506, 5, 3)
    out = [torch.empty(1, 5, 128, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    vs.qk_norm_rope(x[:, :1], x[:, 1:2], out[0], out[1], rope, pos0=1000)
    rope.freq = vs.rope_frequencies(5e5, 64).cuda()
    vs.qk_norm_rope(x[:, :1], x[:, 1:2], out[2], out[3], rope, pos0=1000)
    vs.qk_norm_rope(x[:, :1], x[:, 1:2], out[0], out[1], vs.Rope(vs.rope_frequencies(5e5, 64).cuda(), 1), pos0=1000)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
