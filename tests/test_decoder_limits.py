"""The ends of what a quantised decoder layer's calls accept, without a GPU: sizes are those of the formulas, or refused."""
import ctypes

import pytest

from paper_2304_09049_amd import binding as dg

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
RANGE, BUFFER = 3, 4


def cache_bytes(pages, page_size, heads, dim, bits):
    """By the layout that the header states, in Python's whole numbers."""
    return pages * heads * page_size * (2 * dim * bits // 8 + (8 if bits == 8 else 16))


@pytest.mark.parametrize("desc", [(1, 2097152, 1, 256, 8), (1, 4194304, 1, 128, 8), (1, 4194304, 1, 256, 4), (1, 1048576, 1, 256, 8), (3, 1048576, 5, 256, 8),
                                  (1, 2097136, 7, 256, 4), (1, 14913072, 2, 64, 4), (1 << 20, 1024, 8, 128, 8)])
def test_sizes_of_large_caches(desc):
    assert dg.dg_cache_bytes(dg.cache_desc(*desc)) == cache_bytes(*desc)


@pytest.mark.parametrize("desc", [(1, 1 << 26, 1, 64, 8), (1, 4194304, 1, 256, 8), (1 << 26, 16, 1 << 28, 256, 8), (1 << 26, 16, (1 << 31) - 1, 64, 4),
                                  ((1 << 27) - 1, 16, 1 << 27, 128, 8)])
def test_caches_that_are_too_large(desc):
    d = dg.cache_desc(*desc)
    assert dg.dg_cache_bytes(d) == 0
    status = dg.lib().dg_cache_write(ctypes.byref(d), FAKE, ctypes.c_size_t(-1).value, FAKE, FAKE, 0, 1, 64, 64, 64, 64, FAKE, None)
    assert status == RANGE


def test_a_large_page_needs_its_bytes():
    d = dg.cache_desc(1, 2097152, 1, 256, 8)
    write = lambda n: dg.lib().dg_cache_write(ctypes.byref(d), FAKE, n, None, None, 0, 1, 256, 256, 256, 256, FAKE, None)  # noqa: E731
    assert write(cache_bytes(1, 2097152, 1, 256, 8) - 1) == BUFFER and write(16777216) == BUFFER
    assert write(cache_bytes(1, 2097152, 1, 256, 8)) == 1                  # enough: what is wrong now is a NULL


def test_more_heads_than_a_launch_takes():
    d = dg.cache_desc(1, 16, (1 << 24) + 1, 64, 8)
    size = dg.dg_cache_bytes(d)
    assert size == cache_bytes(1, 16, (1 << 24) + 1, 64, 8)
    assert dg.lib().dg_cache_write(ctypes.byref(d), FAKE, size, FAKE, FAKE, 0, 1, 64, 64, 64, 64, FAKE, None) == RANGE
    assert dg.lib().dg_cache_read(ctypes.byref(d), FAKE, size, FAKE, 1, FAKE, FAKE, 0, None) == RANGE
