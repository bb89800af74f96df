"""Caches whose size or offsets would pass 64 bits: the size does not wrap, and no call takes such a cache."""
import ctypes

import pytest

import paper_2603_04460_amd as vs
from paper_2603_04460_amd import binding

PAGE = 4096 * (1 << 14) * vs.CACHE_BLOCK_BYTES              # bytes of the largest page: 4096 heads, 2^20 tokens


def test_sizes_past_64_bits():
    wraps = -(-2 ** 64 // PAGE)
    assert wraps * PAGE - 2 ** 64 == 1 << 36                # a size that a GPU has
    for pages in (wraps, wraps + 1, 2 * wraps, 2 ** 31 - 1):
        assert vs.cache_bytes(pages, 4096, 1 << 20) == 2 ** 64 - PAGE
    for pages in (wraps - 1, (2 ** 63 - 1) // PAGE, (2 ** 63 - 1) // PAGE + 1):
        assert vs.cache_bytes(pages, 4096, 1 << 20) == pages * PAGE
    assert vs.cache_bytes(2 ** 31 - 1, 3, 1 << 20) == (2 ** 31 - 1) * 3 * (1 << 14) * vs.CACHE_BLOCK_BYTES


@pytest.mark.parametrize("table", [True, False])
def test_calls_refuse_offsets_past_63_bits(table):
    """Told from larger ones by the workspace, which is looked at last: nothing is launched."""
    buf = (ctypes.c_char * 4096)()
    p = (ctypes.addressof(buf) + 15) & ~15
    L = binding._load()
    most = (2 ** 63 - 1) // PAGE
    for pages, attend, other in ((most, -3, None), (most + 1, -2, -2), (-(-2 ** 64 // PAGE), -2, -2), (2 ** 31 - 1, -2, -2)):
        c = ctypes.byref(binding._Cache(p, pages, 4096, 1 << 20, p if table else None, 1))
        assert L.vs_cache_attend(p, c, 1, 4096, 1, p, 1 << 20, 0.1, p, None, None, 0, None) == attend, pages
        if other is not None:
            assert L.vs_cache_write(c, p, p, 1, 1, p, 100, None) == other, pages
            assert L.vs_cache_read(c, 1, 1, p, 100, p, p, None) == other, pages
