"""vs_qk_norm_rope with heads shared out unevenly over workgroups (bounds: test_gpu_norm_rope.py)."""
import numpy as np
import pytest
import torch

import paper_2603_04460_amd as vs
import test_gpu_norm_rope as norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq, hk, rows", [(32, 8, 1000), (33, 11, 1000), (9, 1, 500), (5, 5, 2000), (40, 2, 37), (21, 7, 5000)])
def test_heads_shared_out(hq, hk, rows):
    """Heads that no whole number of workgroups divides: each is there once, none of the neighbouring memory is written."""
    x = norm.packed(hq, rows, hq + 2 * hk)
    freq, w = vs.rope_frequencies(1e6), norm.weight(8)
    whole = [torch.full((h + 2, rows, 128), 9.5, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk)]
    out = [t[1:-1] for t in whole]
    vs.qk_norm_rope(x[:, :hq], x[:, hq:hq + hk], out[0], out[1], vs.Rope(freq.cuda(), 1), v=x[:, hq + hk:], v_out=out[2], w_q=w, w_k=w, pos0=11)
    pos = 11 + np.arange(rows)[None]
    norm.check(out[0][None], norm.heads_first(x[:, :hq], 1, rows), w, 1e-6, freq.numpy(), pos, 1)
    norm.check(out[1][None], norm.heads_first(x[:, hq:hq + hk], 1, rows), w, 1e-6, freq.numpy(), pos, 1)
    assert torch.equal(out[2], x[:, hq + hk:].transpose(0, 1))
    assert all(bool((t[0] == 9.5).all() and (t[-1] == 9.5).all()) for t in whole)
