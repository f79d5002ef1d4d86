"""The paged cache's C ABI without a GPU: every function that
include/wm_cache.h declares is exported and bound, sizes are what the header
says, and host-side argument checks return the documented codes before any
device work (the addresses passed here are never dereferenced)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wm_cache.h")
LIB = os.path.join(ROOT, "paper_2607_10389_amd", "libwm.so")

OK, INVALID, CAPACITY, WORKSPACE, UNSUPPORTED = 0, -1, -2, -4, -5
A = 0x7f0000001000


@pytest.fixture(scope="module")
def cache():
    if not os.path.exists(LIB):
        pytest.skip("libwm.so is not built")
    from paper_2607_10389_amd import _cache
    return _cache


def declared():
    text = open(HEADER).read()
    return re.findall(r"^\s*(?:wm_status|uint64_t)\s*(wm_\w+)\s*\(", text, flags=re.M)


def test_every_declared_symbol_is_exported_and_bound(cache):
    names = declared()
    assert len(names) == len(set(names)) == 7
    for name in names:
        assert hasattr(cache.LIB, name), name
    assert sorted(cache.EXPORTS) == sorted(names)


def desc(cache, **kw):
    d = dict(k=A, v=A + 4096, k_scale=A, v_scale=A, k_stride=8 * 64 * 128, v_stride=8 * 64 * 128,
             k_scale_stride=8, v_scale_stride=8, n_blocks=10, n_heads=8, block_tokens=64,
             head_dim=128, format=1, flags=0)
    d.update(kw)
    return cache.Cache(**d)


def rows(cache, **kw):
    d = dict(ptr=A, row_stride=1024, head_stride=128, dtype=1, flags=0)
    d.update(kw)
    return cache.Rows(**d)


BAD_CACHE = [
    (dict(k=A + 8), INVALID), (dict(v=None), INVALID), (dict(k_scale=None), INVALID),
    (dict(v_scale=A + 2), INVALID), (dict(n_blocks=0), INVALID), (dict(n_blocks=1 << 31), INVALID),
    (dict(n_heads=0), INVALID), (dict(n_heads=65536), INVALID), (dict(format=3), INVALID),
    (dict(flags=1), INVALID), (dict(k_stride=8 * 64 * 128 - 16), INVALID),
    (dict(v_stride=8 * 64 * 128 + 8), INVALID), (dict(k_scale_stride=7), INVALID),
    (dict(block_tokens=48), UNSUPPORTED), (dict(block_tokens=8), UNSUPPORTED),
    (dict(block_tokens=512), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED),
    (dict(head_dim=320), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache_descriptions_that_are_refused(cache, kw, status):
    r = rows(cache)
    assert cache.LIB.wm_cache_append(desc(cache, **kw), r, r, A, A, 2, 5, None, None) == status
    assert cache.LIB.wm_cache_attend(desc(cache, **kw), r, r, None, 8, A, 4, 4, A, A, 2, 5, 256,
                                     1.0, 0, None, None, 0, None) == status


def test_append_argument_checks(cache):
    c, r, fn = desc(cache), rows(cache), cache.LIB.wm_cache_append
    assert fn(None, r, r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, None, r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, rows(cache, dtype=3), r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, r, rows(cache, dtype=2), A, A, 2, 5, None, None) == INVALID  # k and v differ
    assert fn(c, rows(cache, flags=1), r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, rows(cache, ptr=A + 1), r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, rows(cache, ptr=None), r, A, A, 2, 5, None, None) == INVALID
    assert fn(c, r, r, None, A, 2, 5, None, None) == INVALID
    assert fn(c, r, r, A + 4, A, 2, 5, None, None) == INVALID
    assert fn(c, r, r, A, None, 2, 5, None, None) == INVALID
    assert fn(c, r, r, A, A, 2, 5, A + 2, None) == INVALID
    # nothing to store: no device work
    assert fn(c, r, r, None, None, 0, 5, None, None) == OK
    assert fn(c, r, r, None, None, 2, 0, None, None) == OK


def test_attend_argument_checks(cache):
    c, r = desc(cache), rows(cache)

    def call(q=r, out=r, lse=None, hq=8, table=A, stride=4, width=4, lens=A, starts=A, n=2,
             tokens=5, most=256, scale=1.0, window=0, verdict=None, ws=None, ws_bytes=0):
        return cache.LIB.wm_cache_attend(c, q, out, lse, hq, table, stride, width, lens, starts,
                                         n, tokens, most, scale, window, verdict, ws, ws_bytes,
                                         None)
    assert call(q=None) == INVALID
    assert call(out=rows(cache, dtype=2)) == INVALID
    assert call(hq=12) == INVALID  # no multiple of the key heads
    assert call(hq=0) == INVALID
    assert call(lse=A + 2) == INVALID
    assert call(table=None) == INVALID
    assert call(stride=3) == INVALID
    assert call(width=1 << 26, stride=1 << 26) == INVALID  # tokens beyond 32 bits
    assert call(lens=None) == INVALID
    assert call(starts=A + 2) == INVALID
    assert call(scale=float("nan")) == INVALID
    assert call(scale=float("inf")) == INVALID
    assert call(window=1 << 31) == INVALID
    assert call(most=1 << 31) == INVALID
    assert call(verdict=A + 1) == INVALID
    need = cache.LIB.wm_attend_ws_bytes(2, 5, 8, 8, 128, 1 << 17)
    assert need > 0
    big = dict(width=2048, stride=2048, most=1 << 17)
    assert call(**big) == WORKSPACE
    assert call(ws=A, ws_bytes=need - 1, **big) == WORKSPACE
    assert call(ws=A + 8, ws_bytes=need, **big) == WORKSPACE
    assert call(n=0) == OK and call(tokens=0) == OK


def test_page_tables_argument_checks(cache):
    def call(old=A, new=A, n=3, bt=64, table=A, stride=4, width=4, ring=A, cap=100, p0=A,
             p1=A + 8, slots=A, slot_cap=10, starts=A, verdict=A):
        return cache.LIB.wm_page_tables(old, new, n, bt, table, stride, width, ring, cap, p0, p1,
                                        slots, slot_cap, starts, verdict, None)
    assert call(bt=24) == UNSUPPORTED
    for kw in (dict(old=None), dict(new=None), dict(table=None), dict(ring=None), dict(cap=0),
               dict(p0=None), dict(p1=None), dict(p1=A), dict(starts=None), dict(verdict=None),
               dict(slots=None), dict(slots=A + 4), dict(stride=3), dict(cap=1 << 31),
               dict(old=A + 1), dict(width=1 << 26, stride=1 << 26), dict(slot_cap=1 << 31)):
        assert call(**kw) == INVALID, kw


def test_pages_argument_checks(cache):
    def table(*pools):
        t = (cache.Pool * max(len(pools), 1))()
        for i, p in enumerate(pools):
            t[i] = cache.Pool(*p)
        return t
    good = (A, 4096, 8192, 10)
    t, lib = table(good, (A, 20, 20, 12)), cache.LIB
    total = 3 * 4096 + 64
    assert lib.wm_flat_pages_bytes(t, 2, 3) == total
    assert lib.wm_flat_pages_bytes(None, 2, 3) == 0
    assert lib.wm_flat_pages_bytes(table((A, 1 << 62, 1 << 62, 1)), 1, 4) == 0
    for flat_first in (False, True):
        def call(t=t, n=2, pages=A, n_pages=3, flat=A, cap=total, verdict=A):
            if flat_first:
                return lib.wm_rehydrate_pages(flat, cap, t, n, pages, n_pages, verdict, None)
            return lib.wm_flatten_pages(t, n, pages, n_pages, flat, cap, verdict, None)
        assert call(cap=total - 1) == CAPACITY
        assert call(t=None) == INVALID
        assert call(n=4097) == INVALID
        assert call(verdict=None) == INVALID
        assert call(pages=None) == INVALID
        assert call(pages=A + 2) == INVALID
        assert call(flat=None) == INVALID
        assert call(flat=A + 8) == INVALID
        for bad in ((A + 2, 4096, 4096, 10), (None, 4096, 4096, 10), (A, 4098, 8192, 10),
                    (A, 4096, 4094, 10), (A, 4096, 2048, 10), (A, 4096, 4096, 0),
                    (A, 0, 0, 10), (A, 4096, 4096, 1 << 31)):
            assert call(t=table(bad), n=1, cap=1 << 40) == INVALID, bad
        # nothing to copy
        assert call(n_pages=0, pages=None, flat=None, cap=0) == OK
        assert call(t=None, n=0, flat=None, cap=0) == OK


def test_workspace_covers_the_split(cache):
    ws = cache.LIB.wm_attend_ws_bytes
    assert ws(0, 0, 8, 8, 128, 100) == 0
    assert ws(64, 64, 8, 32, 128, 64) == 0          # one step: nothing to split
    assert ws(1, 1, 1, 1, 128, 0x7FFFFFFF) > 0      # the longest sequence
    assert ws(1, 4096, 8, 32, 128, 4096) == 0       # a prompt fills the GPU by its rows


def test_binding_refuses_host_tensors(cache):
    import torch
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        cache.page_tables(t, t, 64, t.view(2, 2), t, t, t, t.long(), t, t)
    k = torch.zeros(2, 1, 16, 64, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        cache.cache_desc(k, k.view(2, 1, 64, 16), torch.zeros(2, 1), torch.zeros(2, 1))
    with pytest.raises(ValueError):
        cache.PoolTable([torch.zeros(4, 4)])


def test_binding_refuses_numbers_beyond_32_bits(cache, monkeypatch):
    import torch
    calls = []
    monkeypatch.setattr(cache, "_device", lambda t: t.get_device())
    monkeypatch.setattr(cache, "_run", lambda *args: calls.append(args))
    k = torch.zeros(2, 1, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    v, s = k.view(2, 1, 64, 16), torch.zeros(2, 1)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    one = torch.ones(1, dtype=torch.int32)
    args = (q, k, v, s, s, one[None], one, torch.zeros(2, dtype=torch.int32), torch.zeros_like(q))
    for bad in (dict(window=1 << 32), dict(window=(1 << 32) + 5), dict(window=-1),
                dict(max_len=1 << 32), dict(max_len=-1)):
        with pytest.raises(ValueError):
            cache.cache_attend(*args, **{**dict(max_len=1, scale=1.0), **bad})
    assert not calls
    cache.cache_attend(*args, max_len=1, scale=1.0, window=(1 << 31) - 1)
    assert len(calls) == 1
