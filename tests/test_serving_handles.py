"""A cache and a rotation whose tensors are replaced: the next call takes the new ones, and what does not fit is refused and changes nothing.
On the CPU (tensors of host memory in the place of the GPU's: nothing is launched); test_gpu_cache_growth.py grows a cache on the GPU."""
import pytest
import torch

import paper_2603_04460_amd as vs
from paper_2603_04460_amd import binding


@pytest.fixture(autouse=True)
def host_tensors(monkeypatch):
    def dev(t, dtype, what):
        if not (isinstance(t, torch.Tensor) and t.is_contiguous() and t.dtype == dtype):
            raise TypeError(what)
        return t
    monkeypatch.setattr(binding, "_dev", dev)


def pages(n, heads=2, blocks=1):
    return torch.zeros(n, heads, blocks, vs.CACHE_BLOCK_BYTES, dtype=torch.uint8)


def holds(c):
    """What a call would hand over is what the attributes say."""
    x = c._ref._obj
    table = None if c.table is None else c.table.data_ptr()
    return (x.data, x.pages, x.kv_heads, x.page_size, x.table, x.max_pages) == (c.data.data_ptr(), c.pages, c.kv_heads, c.page_size, table, c.max_pages)


def test_a_cache_that_grows():
    c = vs.Cache(pages(4), torch.zeros(2, 3, dtype=torch.int32))
    assert holds(c) and (c.pages, c.kv_heads, c.page_size, c.max_pages) == (4, 2, 64, 3)
    c.table = torch.ones(2, 7, dtype=torch.int32)
    assert holds(c) and c.max_pages == 7
    c.data = pages(9, 4, 3)
    assert holds(c) and (c.pages, c.kv_heads, c.page_size, c.max_pages) == (9, 4, 192, 7)
    c = vs.Cache(pages(8), max_pages=4)
    c.max_pages = 8
    assert holds(c) and c.max_pages == 8 and c.table is None
    c.data = pages(16)
    assert holds(c) and c.max_pages == 8 and c.pages == 16
    c.table = torch.zeros(1, 5, dtype=torch.int32)
    assert holds(c) and c.max_pages == 5


def test_refused_replacements_change_nothing():
    data, table = pages(4), torch.zeros(2, 3, dtype=torch.int32)
    c = vs.Cache(data, table)
    for name, bad, error in (("table", table.long(), TypeError), ("table", table[:, ::2], TypeError), ("table", table[0], AssertionError),
                             ("table", None, AssertionError), ("data", data[..., 1:], TypeError), ("data", data.short(), TypeError), ("data", data[0], AssertionError),
                             ("max_pages", 5, AssertionError), ("pages", 5, AttributeError), ("kv_heads", 1, AttributeError), ("page_size", 128, AttributeError)):
        with pytest.raises(error):
            setattr(c, name, bad)
        assert c.data is data and c.table is table and holds(c), name


def test_a_rotation_that_is_replaced():
    r = vs.Rope(vs.rope_frequencies(1e6), 1, 1.25)
    x = r._ref._obj
    same = lambda: (r._ref._obj.freq, r._ref._obj.rot_dim, r._ref._obj.pairing, r._ref._obj.magnitude) == (
        r.freq.data_ptr(), 2 * r.freq.numel(), r.pairing, r.magnitude)
    assert same() and x.rot_dim == 128
    r.freq = vs.rope_frequencies(1e6, 64)
    assert same() and r._ref._obj.rot_dim == 64
    r.pairing, r.magnitude = 0, 2.0
    assert same() and (r.pairing, r.magnitude) == (0, 2.0)
    kept = r.freq
    for bad, error in ((kept.float(), TypeError), (kept[None], AssertionError), (kept[::2], TypeError)):
        with pytest.raises(error):
            r.freq = bad
        assert r.freq is kept and same()


class Stream:
    cuda_stream = 77

    def __init__(self, index):
        self.device = torch.device("cuda", index)


def test_streams_of_another_device():
    """The tensors of a call are on the current device, and so has its stream to be."""
    assert binding._stream(Stream(0), 0) == 77 and binding._stream(Stream(3), 3) == 77
    with pytest.raises(ValueError):
        binding._stream(Stream(1), 0)


def test_workspaces_that_hold_less_than_they_say(monkeypatch):
    """A workspace is a contiguous tensor of the current device: nbytes of an expanded one counts memory that it does not have."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)           # where host tensors say that they are
    c = vs.Cache(pages(4), max_pages=4)
    q = torch.zeros(1, 4, 1, 128, dtype=torch.bfloat16)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20)[::2]):
        with pytest.raises(TypeError):
            vs.cache_attend(q, c, torch.zeros_like(q), 300, ws=ws)
