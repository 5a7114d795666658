"""Calls of the decode step that are refused before anything is enqueued, so
that these run without a GPU."""
import ctypes

import pytest

from tests.test_serve_abi import ARG, FAKE, cache, ds   # noqa: F401 (ds: fixture)


@pytest.mark.parametrize("rows", [None, FAKE])
@pytest.mark.parametrize("max_pages", [16, 4096])              # one workgroup's selection, and chunks
@pytest.mark.parametrize("src,dst", [(0x4000, 0x4000), (0x4000, 0x4000 + 4 * 7), (0x4000 + 4 * 3, 0x4000)])
def test_evict_lengths_apart(ds, rows, max_pages, src, dst):   # noqa: F811
    """The new lengths may not be the old ones' array, nor part of it: 8
    requests, 4 rows."""
    p = ds.EvictParams(1, 1, 0, 0, 1 << 20, 1 << 20)
    a, b = cache(ds, max_pages=max_pages, len=src), cache(ds, max_pages=max_pages, len=dst)
    st = ds.lib.ds_cache_evict(ctypes.byref(a), ctypes.byref(b), ctypes.byref(p), 4, rows, FAKE, FAKE, FAKE, FAKE, 0x100000, 1 << 40, 0, None)
    assert st == ARG
