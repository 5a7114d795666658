"""The decode step's C entry points: exported as the header declares them, and
refusing bad host arguments before any HIP call (so these run without a GPU)."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
FAKE, WS = 0x1000, 0x100000          # never dereferenced
OK, NULL, ARG, SIZE, WORKSPACE, ALIGN = 0, -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def ds():
    from paper_2606_02982_amd import driftsched
    return driftsched


def cache(ds, **kw):
    c = ds.KvCache(FAKE, FAKE, None, None, FAKE, FAKE, 8, 16, 128, 16, 2, 64, 16 * 128, 128, 64, 2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_exports_every_declared_symbol(ds):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "driftsched_serve.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ds_[a-z_]+)\s*\(", src)))
    assert names == ["ds_cache_evict", "ds_decode_attention", "ds_decode_workspace_bytes", "ds_evict_workspace_bytes",
                     "ds_verify_draft", "ds_verify_workspace_bytes"]
    for name in names:
        assert hasattr(ds.lib, name), name


def decode(ds, c=None, n_rows=4, rows=FAKE, q=FAKE, out=FAKE, mass=None, ws=WS, ws_bytes=1 << 40, flags=0, **kw):
    p = ds.DecodeParams(8, 1, 2, 512, 512, 64, 0.125, 0, 0, 0, 256)
    for k, v in kw.items():
        setattr(p, k, v)
    c = cache(ds) if c is None else c
    return ds.lib.ds_decode_attention(ctypes.byref(c), ctypes.byref(p), n_rows, rows, q, out, mass, ws, ws_bytes, flags, None)


@pytest.mark.parametrize("field,value,status", [
    ("type", 0, ARG), ("type", 4, ARG), ("type", 1, ARG), ("head_dim", 0, ARG), ("head_dim", 12, ARG), ("head_dim", 264, ARG),
    ("n_kv", 0, ARG), ("n_kv", 3, ARG), ("page_size", 0, ARG), ("n_pages", 0, ARG), ("max_pages", 0, ARG), ("n_requests", 0, ARG),
    ("page_stride", 4, ALIGN), ("token_stride", 4, ALIGN), ("head_stride", 4, ALIGN), ("max_pages", 1 << 27, SIZE), ("k", None, NULL),
    ("v", None, NULL), ("table", None, NULL), ("len", None, NULL), ("k", 0x1008, ALIGN), ("v", 0x1004, ALIGN), ("table", 0x1002, ALIGN),
    ("len", 0x1001, ALIGN), ("k_scale", FAKE, ARG), ("v_scale", FAKE, ARG)])
def test_cache_errors(ds, field, value, status):
    assert decode(ds, cache(ds, **{field: value})) == status
    if field not in ("type", "n_kv"):
        p = ds.EvictParams(1, 1, 0, 0, 256, 256)
        good, bad = cache(ds), cache(ds, **{field: value})
        for a, b in ((bad, good), (good, bad)):
            st = ds.lib.ds_cache_evict(ctypes.byref(a), ctypes.byref(b), ctypes.byref(p), 4, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, 0, None)
            assert st == status


@pytest.mark.parametrize("kw,status", [
    (dict(n_q=0), ARG), (dict(n_q=3), ARG), (dict(n_tokens=0), ARG), (dict(n_tokens=17), ARG), (dict(q_type=0), ARG), (dict(q_type=1), ARG),
    (dict(q_type=3), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(scale=1e39), ARG),
    (dict(max_len=257), ARG), (dict(q_row_stride=4), ALIGN), (dict(q_token_stride=4), ALIGN), (dict(q_head_stride=4), ALIGN),
    (dict(n_q=2 * 1025), SIZE), (dict(n_q=2 * 512, n_tokens=3), SIZE), (dict(mass=FAKE, mass_len=255), ARG),
    (dict(n_rows=9, rows=None), ARG), (dict(n_rows=0xFFFFFFFF), SIZE), (dict(q=None), NULL), (dict(out=None), NULL),
    (dict(q=0x1008), ALIGN), (dict(out=0x1002), ALIGN), (dict(rows=0x1001), ALIGN), (dict(mass=0x1002), ALIGN),
    (dict(ws=None, flags=1), WORKSPACE), (dict(ws=0x100010, flags=1), WORKSPACE), (dict(ws_bytes=255, flags=1), WORKSPACE),
    (dict(mass=FAKE, ws=None), WORKSPACE), (dict(n_rows=0), OK)])
def test_decode_errors(ds, kw, status):
    assert decode(ds, **kw) == status


def test_decode_null_structs(ds):
    c, p = cache(ds), ds.DecodeParams(8, 1, 2, 512, 512, 64, 0.125, 0, 0, 0, 256)
    assert ds.lib.ds_decode_attention(None, ctypes.byref(p), 4, FAKE, FAKE, FAKE, None, WS, 1 << 40, 0, None) == NULL
    assert ds.lib.ds_decode_attention(ctypes.byref(c), None, 4, FAKE, FAKE, FAKE, None, WS, 1 << 40, 0, None) == NULL
    assert ds.lib.ds_decode_workspace_bytes(None, ctypes.byref(p), 4, 0) == 0


def test_decode_workspace(ds):
    """Grows with the rows and the weights' sum; a byte less is refused."""
    c, p = cache(ds, max_pages=4096), ds.DecodeParams(8, 2, 2, 1024, 512, 64, 0.125, 0, 0, 0, 65536)
    f = lambda n, m: ds.lib.ds_decode_workspace_bytes(ctypes.byref(c), ctypes.byref(p), n, m)   # noqa: E731
    assert f(0, 0) == 256 and f(1, 0) > 256 and f(1, 1) > f(1, 0) and f(64, 1) > f(8, 1)
    for m in (None, FAKE):
        need = f(4, m is not None)
        assert ds.lib.ds_decode_attention(ctypes.byref(c), ctypes.byref(p), 4, FAKE, FAKE, FAKE, m, WS, need - 1, 0, None) == WORKSPACE
    # weights of more than 2^24 tokens are not gathered; with a window they need not be
    huge, p = cache(ds, max_pages=(1 << 20) + 16), ds.DecodeParams(8, 2, 2, 1024, 512, 64, 0.125, 0, 0, 0, 1 << 26)
    g = lambda m: ds.lib.ds_decode_workspace_bytes(ctypes.byref(huge), ctypes.byref(p), 1, m)   # noqa: E731
    assert g(0) > 256 and g(1) == 0
    assert ds.lib.ds_decode_attention(ctypes.byref(huge), ctypes.byref(p), 1, FAKE, FAKE, FAKE, FAKE, WS, 1 << 50, 0, None) == SIZE
    p.window = 4096
    assert g(1) > 256
    # 8-bit caches go with either query type
    for t in (1, 2):
        q = ds.DecodeParams(8, 1, t, 512, 512, 64, 0.125, 0, 0, 0, 0)
        assert ds.lib.ds_decode_workspace_bytes(ctypes.byref(cache(ds, type=3)), ctypes.byref(q), 4, 0) >= 256
    assert ds.lib.ds_decode_workspace_bytes(ctypes.byref(cache(ds, type=3, head_dim=72)), ctypes.byref(q), 4, 0) == 0


@pytest.mark.parametrize("field,value", [("page_size", 8), ("n_kv", 4), ("head_dim", 32), ("type", 1), ("page_stride", 64), ("token_stride", 64),
                                         ("head_stride", 8)])
def test_evict_needs_one_layout(ds, field, value):
    p = ds.EvictParams(1, 1, 0, 0, 256, 256)
    st = ds.lib.ds_cache_evict(ctypes.byref(cache(ds)), ctypes.byref(cache(ds, **{field: value})), ctypes.byref(p), 4, FAKE, FAKE, FAKE, FAKE,
                               FAKE, None, 0, 0, None)
    assert st == ARG


def test_evict_errors(ds):
    def call(n=4, rows=FAKE, budget=FAKE, mass=FAKE, out=FAKE, kept=FAKE, flags=0, ws=WS, ws_bytes=1 << 40, dst=None, **kw):
        p = ds.EvictParams(1, 1, 0, 0, 256, 256)
        for k, v in kw.items():
            setattr(p, k, v)
        return ds.lib.ds_cache_evict(ctypes.byref(cache(ds)), ctypes.byref(dst or cache(ds)), ctypes.byref(p), n, rows, budget, mass, out, kept,
                                     ws, ws_bytes, flags, None)
    assert call(n=0) == OK
    assert call(n=9) == ARG                                    # more rows than dst holds
    assert ds.lib.ds_evict_workspace_bytes(*map(ctypes.byref, (cache(ds, n_requests=1 << 28),) * 2 + (ds.EvictParams(1, 1, 0, 0, 256, 256),)),
                                           1 << 28) == 0       # more workgroups than a launch takes
    assert call(mass_len=255) == ARG and call(max_len=300) == ARG
    assert call(n=9, rows=None, dst=cache(ds, n_requests=20)) == ARG
    assert call(budget=None) == NULL and call(mass=None) == NULL and call(out=None) == NULL and call(kept=None) == NULL
    assert call(budget=0x1004) == ALIGN and call(kept=0x1002) == ALIGN and call(rows=0x1002) == ALIGN
    assert call(flags=1, ws=None) == WORKSPACE and call(flags=1, ws_bytes=255) == WORKSPACE and call(flags=1, ws=0x100010) == WORKSPACE
    assert ds.lib.ds_cache_evict(ctypes.byref(cache(ds)), ctypes.byref(cache(ds)), None, 4, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, 0, None) == NULL


def test_evict_workspace(ds):
    """Nothing but the flag for short requests, chunks for long ones."""
    p = ds.EvictParams(1, 1, 0, 0, 1 << 24, 1 << 24)
    need = lambda c, n: ds.lib.ds_evict_workspace_bytes(ctypes.byref(c), ctypes.byref(c), ctypes.byref(p), n)   # noqa: E731
    assert need(cache(ds, max_pages=1536), 4) == 256 and need(cache(ds, max_pages=1537), 4) > 256
    assert need(cache(ds, max_pages=1 << 20), 4) > need(cache(ds, max_pages=4096), 4) > need(cache(ds, max_pages=4096), 2)
    assert need(cache(ds, type=0), 4) == 0 and ds.lib.ds_evict_workspace_bytes(None, None, ctypes.byref(p), 4) == 0
    big = cache(ds, max_pages=4096)
    for ws_bytes, status in ((need(big, 4) - 1, WORKSPACE),):
        assert ds.lib.ds_cache_evict(ctypes.byref(big), ctypes.byref(big), ctypes.byref(p), 4, FAKE, FAKE, FAKE, FAKE, FAKE, WS, ws_bytes, 0,
                                     None) == status


def test_verify_errors(ds):
    def call(n=4, rows=None, target=FAKE, draft=FAKE, tokens=FAKE, nd=None, u=FAKE, us=FAKE, out=FAKE, em=FAKE, ob=FAKE, ln=None, ws=WS,
             ws_bytes=1 << 40, flags=0, **kw):
        p = ds.VerifyParams(3, 1000, 8, 0, 4000, 1000, 3000, 1000)
        for k, v in kw.items():
            setattr(p, k, v)
        return ds.lib.ds_verify_draft(ctypes.byref(p), n, rows, target, draft, tokens, nd, u, us, out, em, ob, ln, ws, ws_bytes, flags, None)
    assert call(n=0) == OK
    for kw, status in ((dict(type=3), ARG), (dict(type=-1), ARG), (dict(n_drafts=64), ARG), (dict(vocab=0), ARG),
                       (dict(vocab=(1 << 24) + 1), SIZE), (dict(n=0xFFFFFFFF), SIZE), (dict(n=9), ARG), (dict(target=None), NULL),
                       (dict(tokens=None), NULL), (dict(u=None), NULL), (dict(us=None), NULL), (dict(out=None), NULL), (dict(em=None), NULL),
                       (dict(target=0x1002), ALIGN), (dict(draft=0x1002), ALIGN), (dict(tokens=0x1001), ALIGN), (dict(nd=0x1001), ALIGN),
                       (dict(ob=0x1002), ALIGN), (dict(ln=0x1002), ALIGN), (dict(rows=0x1002), ALIGN), (dict(ws=None), WORKSPACE),
                       (dict(ws_bytes=256), WORKSPACE)):
        assert call(**kw) == status, kw
    assert ds.lib.ds_verify_workspace_bytes(None, 4) == 0
    p = ds.VerifyParams(3, 100000, 8, 0, 4000, 1000, 3000, 1000)
    assert ds.lib.ds_verify_workspace_bytes(ctypes.byref(p), 40) > ds.lib.ds_verify_workspace_bytes(ctypes.byref(p), 4) > 256


def test_binding_refuses(ds):
    """Tensors that are not on the device, of other types or shapes."""
    k = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    table, lens = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for bad in (lambda: ds.kv_cache(k, k, table, lens),                               # not on the device
                lambda: ds.kv_cache(k, k[:, :8], table, lens), lambda: ds.kv_cache(k.float(), k.float(), table, lens),
                lambda: ds.kv_cache(k, k.half(), table, lens), lambda: ds.kv_cache(k, k, table, lens[:1]),
                lambda: ds.kv_cache(k, k, table[0], lens), lambda: ds.kv_cache(k.transpose(2, 3), k.transpose(2, 3), table, lens),
                lambda: ds.verify_draft(torch.zeros((2, 3, 8)), None, torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 2)), torch.zeros(2)),
                lambda: ds.verify_draft(torch.zeros((2, 0, 8)), None, torch.zeros((2, 0), dtype=torch.int32), torch.zeros((2, 0)), torch.zeros(2)),
                lambda: ds.verify_draft(torch.zeros((2, 3, 8)), torch.zeros((2, 3, 8)), torch.zeros((2, 2), dtype=torch.int32),
                                        torch.zeros((2, 2)), torch.zeros(2))):
        with pytest.raises(ValueError):
            bad()
