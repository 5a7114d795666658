"""Calls of the decode step that are refused before anything is enqueued, so
that these run without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("value", [-1, -(1 << 31), 1 << 32, (1 << 32) + 5, 2.5, float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["window", "sinks", "max_len"])
def test_attention_counts(ds, name, value):   # noqa: F811
    """Counts that 32 bits do not hold are refused, before the tensors are
    looked at, and not taken modulo 2^32."""
    with pytest.raises(ValueError, match=name):
        ds.decode_attention(None, None, **{name: value})


@pytest.mark.parametrize("value", [-1, -(1 << 31), 1 << 32, (1 << 32) + 5, 2.5, float("nan"), float("-inf")])
@pytest.mark.parametrize("name", ["sinks", "recent", "slack", "max_len"])
def test_eviction_counts(ds, name, value):   # noqa: F811
    with pytest.raises(ValueError, match=name):
        ds.cache_evict(None, None, None, None, **{name: value})


@pytest.mark.parametrize("kind", [np.int64, np.uint32, float, bool, torch.tensor])
def test_counts_of_other_types(ds, kind):   # noqa: F811
    """Whole numbers of another type go on to the tensors' checks."""
    q = torch.zeros((1, 1, 1, 8), dtype=torch.float32)
    with pytest.raises(AttributeError):
        ds.decode_attention(q, None, window=kind(1), sinks=kind(1), max_len=kind(1))
    with pytest.raises(ValueError, match="device"):
        ds.cache_evict(None, None, q, None, sinks=kind(1), recent=kind(1), slack=kind(1), max_len=kind(1))
