"""ctypes binding of libwm's paged 8-bit attention cache (include/wm_cache.h).

Argument marshalling and checks only, as in ``_wm``: the work runs in the HIP
kernels of libwm.so.  A layer's cache is four tensors: key codes
[blocks, heads, block_tokens, dim] and value codes [blocks, heads, dim,
block_tokens] of torch.float8_e4m3fn or torch.float8_e5m2, and their float32
scales [blocks, heads]; only the stride between blocks is free.  Calls run on
the tensors' device and, without a ``stream``, on its current stream.
"""
from __future__ import annotations

import ctypes

import torch

from ._wm import LIB, _check

C_LENGTH, C_POOL, C_SLOTS, C_PAGE = 1, 2, 4, 8

WM_BF16, WM_FP16 = 1, 2
WM_E4M3, WM_E5M2 = 1, 2
WM_MAX_POOLS = 4096

# every symbol declared in include/wm_cache.h
EXPORTS = (
    "wm_page_tables", "wm_cache_append", "wm_cache_attend", "wm_attend_ws_bytes",
    "wm_flat_pages_bytes", "wm_flatten_pages", "wm_rehydrate_pages",
)

_DTYPE = {torch.bfloat16: WM_BF16, torch.float16: WM_FP16}
_FORMAT = {torch.float8_e4m3fn: WM_E4M3, torch.float8_e5m2: WM_E5M2}


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("k_stride", ctypes.c_uint64), ("v_stride", ctypes.c_uint64),
                ("k_scale_stride", ctypes.c_uint64), ("v_scale_stride", ctypes.c_uint64),
                ("n_blocks", ctypes.c_uint32), ("n_heads", ctypes.c_uint32),
                ("block_tokens", ctypes.c_uint32), ("head_dim", ctypes.c_uint32),
                ("format", ctypes.c_uint32), ("flags", ctypes.c_uint32)]


class Rows(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("row_stride", ctypes.c_uint64),
                ("head_stride", ctypes.c_uint64), ("dtype", ctypes.c_uint32),
                ("flags", ctypes.c_uint32)]


class Pool(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("page_bytes", ctypes.c_uint64),
                ("stride", ctypes.c_uint64), ("n_blocks", ctypes.c_uint64)]


def _declare():
    vp, u64, u32, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int32
    cp, rp, pp = ctypes.POINTER(Cache), ctypes.POINTER(Rows), ctypes.POINTER(Pool)
    sig = {
        "wm_page_tables": ([vp, vp, u32, u32, vp, u64, u32, vp, u32, vp, vp, vp, u64, vp, vp,
                            vp], i32),
        "wm_cache_append": ([cp, rp, rp, vp, vp, u32, u32, vp, vp], i32),
        "wm_cache_attend": ([cp, rp, rp, vp, u32, vp, u64, u32, vp, vp, u32, u32, u32,
                             ctypes.c_float, u32, vp, vp, u64, vp], i32),
        "wm_attend_ws_bytes": ([u32, u32, u32, u32, u32, u32], u64),
        "wm_flat_pages_bytes": ([pp, u32, u32], u64),
        "wm_flatten_pages": ([pp, u32, vp, u32, vp, u64, vp, vp], i32),
        "wm_rehydrate_pages": ([vp, u64, pp, u32, vp, u32, vp, vp], i32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(LIB, name)
        fn.argtypes, fn.restype = args, res


_declare()


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _vec(t, dtype, dev, name, n=None):
    """Address of a dense one-dimensional tensor (of at least n entries)."""
    _need(t.dtype == dtype and t.dim() == 1 and (t.numel() <= 1 or t.stride(0) == 1),
          f"{name} is a dense vector of {dtype}")
    _need(t.device == dev, f"{name} is on {t.device}, not on {dev}")
    _need(n is None or t.numel() >= n, f"{name} has fewer than {n} entries")
    return t.data_ptr()


def _word(t, dev):
    """Address of the verdict word (None -> NULL)."""
    if t is None:
        return None
    _need(t.dtype in (torch.int32, torch.uint32) and t.numel() >= 1 and t.device == dev,
          "verdict is a 32-bit word on the same device")
    return t.data_ptr()


def _device(t):
    _need(t.is_cuda, "libwm takes device tensors")
    return t.device


def _run(where, dev, stream, fn, *args):
    """fn(*args, stream) on dev: a stream belongs to a device, and a kernel is
    launched on the current one."""
    s = stream if stream is not None else torch.cuda.current_stream(dev)
    _need(s.device == dev, f"the stream is of {s.device}, the tensors are on {dev}")
    if dev.index == torch.cuda.current_device():
        return _check(fn(*args, s.cuda_stream), where)
    with torch.cuda.device(dev):
        return _check(fn(*args, s.cuda_stream), where)


def cache_desc(k_cache, v_cache, k_scale, v_scale) -> Cache:
    """The library's description of one layer's cache."""
    dev = _device(k_cache)
    _need(k_cache.dtype in _FORMAT and v_cache.dtype == k_cache.dtype,
          "key and value codes are of one 8-bit float type")
    _need(k_cache.dim() == 4 and v_cache.dim() == 4, "codes are [blocks, heads, .., ..]")
    n, h, bt, d = k_cache.shape
    _need(v_cache.shape == (n, h, d, bt), "value codes are [blocks, heads, dim, block_tokens]")
    ks, vs = k_cache.stride(), v_cache.stride()
    _need((h == 1 or (ks[1] == bt * d and vs[1] == bt * d)) and ks[2] == d and vs[2] == bt
          and ks[3] == 1 and vs[3] == 1, "a block's codes are dense")
    for s in (k_scale, v_scale):
        _need(s.dtype == torch.float32 and s.shape == (n, h) and (h == 1 or s.stride(1) == 1),
              "scales are float32 [blocks, heads], dense within a block")
    _need(v_cache.device == dev and k_scale.device == dev and v_scale.device == dev,
          "a cache's tensors are on one device")
    one = n == 1  # the stride of a single block says nothing
    return Cache(k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                 h * bt * d if one else ks[0], h * bt * d if one else vs[0],
                 h if one else k_scale.stride(0), h if one else v_scale.stride(0),
                 n, h, bt, d, _FORMAT[k_cache.dtype], 0)


def _rows(t, heads, dim, name) -> Rows:
    _need(t.dtype in _DTYPE and t.dim() == 3 and t.shape[1] == heads and t.shape[2] == dim
          and t.stride(2) == 1, f"{name} is [tokens, {heads}, {dim}] of bfloat16 or float16, "
          "its vectors dense")
    return Rows(t.data_ptr(), t.stride(0), t.stride(1), _DTYPE[t.dtype], 0)


def page_tables(old_len, new_len, block_tokens, block_table, free_ring, pool_in, pool_out,
                slot_map, q_start, verdict, stream=None):
    """Block tables and slot maps of a step that takes request r from
    old_len[r] to new_len[r] tokens (wm_page_tables).  block_table is
    [requests, max_blocks], free_ring the ring of free blocks, pool_in and
    pool_out {first place, count}; slot_map is int64, the rest int32."""
    dev, i32, n = _device(old_len), torch.int32, old_len.numel()
    _need(block_table.dtype == i32 and block_table.dim() == 2 and block_table.shape[0] >= n
          and (block_table.shape[1] <= 1 or block_table.stride(1) == 1)
          and block_table.device == dev, "block_table is int32 [requests, max_blocks]")
    width = block_table.shape[1]
    stride = block_table.stride(0) if block_table.shape[0] > 1 else width
    return _run("wm_page_tables", dev, stream, LIB.wm_page_tables,
                _vec(old_len, i32, dev, "old_len"), _vec(new_len, i32, dev, "new_len", n), n,
                block_tokens, block_table.data_ptr(), stride, width,
                _vec(free_ring, i32, dev, "free_ring"), free_ring.numel(),
                _vec(pool_in, i32, dev, "pool_in", 2), _vec(pool_out, i32, dev, "pool_out", 2),
                _vec(slot_map, torch.int64, dev, "slot_map"), slot_map.numel(),
                _vec(q_start, i32, dev, "q_start", n + 1), _word(verdict, dev))


def cache_append(k, v, k_cache, v_cache, k_scale, v_scale, slot_map, q_start, verdict=None,
                 stream=None):
    """Store new keys and values [tokens, heads, dim] where slot_map says
    (wm_cache_append); q_start has an entry per request and one more."""
    c = cache_desc(k_cache, v_cache, k_scale, v_scale)
    dev, n = k_cache.device, k.shape[0]
    kr, vr = _rows(k, c.n_heads, c.head_dim, "k"), _rows(v, c.n_heads, c.head_dim, "v")
    _need(v.shape[0] == n and v.dtype == k.dtype and k.device == dev and v.device == dev,
          "k and v have the same tokens, type and device as the cache")
    _need(q_start.numel() >= 1, "q_start has an entry per request and one more")
    return _run("wm_cache_append", dev, stream, LIB.wm_cache_append, c, kr, vr,
                _vec(slot_map, torch.int64, dev, "slot_map", n),
                _vec(q_start, torch.int32, dev, "q_start"), q_start.numel() - 1, n,
                _word(verdict, dev))


def attend_ws_bytes(q, k_cache, lens, max_len: int) -> int:
    """Workspace bytes of cache_attend for queries, caches and lengths of
    these shapes."""
    return int(LIB.wm_attend_ws_bytes(lens.numel(), q.shape[0], k_cache.shape[1], q.shape[1],
                                      k_cache.shape[3], max_len))


def cache_attend(q, k_cache, v_cache, k_scale, v_scale, block_table, lens, q_start, out, ws=None,
                 *, max_len: int, scale: float, window: int = 0, lse=None, verdict=None,
                 stream=None):
    """Attention of q [tokens, query heads, dim] over the cache into out
    (wm_cache_attend).  lens counts the new tokens; ws holds at least
    attend_ws_bytes()."""
    c = cache_desc(k_cache, v_cache, k_scale, v_scale)
    dev, i32, n = k_cache.device, torch.int32, q.shape[0]
    hq = q.shape[1] if q.dim() == 3 else 0
    qr, outr = _rows(q, hq, c.head_dim, "q"), _rows(out, hq, c.head_dim, "out")
    _need(out.shape[0] == n and out.dtype == q.dtype and q.device == dev and out.device == dev,
          "out has the tokens, type and device of q")
    n_req = lens.numel()
    _need(block_table.dtype == i32 and block_table.dim() == 2 and block_table.shape[0] >= n_req
          and (block_table.shape[1] <= 1 or block_table.stride(1) == 1)
          and block_table.device == dev, "block_table is int32 [requests, max_blocks]")
    width = block_table.shape[1]
    stride = block_table.stride(0) if block_table.shape[0] > 1 else width
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.shape == (n, hq) and lse.is_contiguous()
              and lse.device == dev, "lse is dense float32 [tokens, query heads]")
    if ws is not None:
        _need(ws.device == dev and ws.is_contiguous(), "ws is a dense tensor on the same device")
    return _run("wm_cache_attend", dev, stream, LIB.wm_cache_attend, c, qr, outr,
                None if lse is None else lse.data_ptr(), hq, block_table.data_ptr(), stride,
                width, _vec(lens, i32, dev, "lens"),
                _vec(q_start, i32, dev, "q_start", n_req + 1), n_req, n, max_len, scale, window,
                _word(verdict, dev), None if ws is None else ws.data_ptr(),
                0 if ws is None else ws.numel() * ws.element_size())


class PoolTable:
    """Host table of pools [blocks, ...] (device tensors whose pages are dense;
    the stride between pages is free); build it once to move the pages of many
    sessions."""

    def __init__(self, pools):
        self.n = len(pools)
        self.t = (Pool * max(self.n, 1))()
        self.device = _device(pools[0]) if self.n else None
        for i, x in enumerate(pools):
            _need(x.is_cuda and x.dim() >= 1 and x.shape[0] > 0 and x[0].is_contiguous()
                  and x.device == self.device,
                  "pools are device tensors [blocks, ...] with dense pages")
            page = x[0].numel() * x.element_size()
            self.t[i].ptr, self.t[i].page_bytes = x.data_ptr(), page
            self.t[i].stride = x.stride(0) * x.element_size() if x.shape[0] > 1 else page
            self.t[i].n_blocks = x.shape[0]


def _pools(pools) -> PoolTable:
    return pools if isinstance(pools, PoolTable) else PoolTable(pools)


def flat_pages_bytes(pools, n_pages: int) -> int:
    tab = _pools(pools)
    return int(LIB.wm_flat_pages_bytes(tab.t, tab.n, n_pages))


def flatten_pages(pools, pages, flat, verdict, stream=None):
    """Gather the pools' listed pages into flat (wm_flatten_pages)."""
    tab, dev = _pools(pools), _device(flat)
    _need(tab.device in (None, dev) and flat.is_contiguous(), "flat is dense, on the pools' device")
    return _run("wm_flatten_pages", dev, stream, LIB.wm_flatten_pages, tab.t, tab.n,
                _vec(pages, torch.int32, dev, "pages"), pages.numel(), flat.data_ptr(),
                flat.numel() * flat.element_size(), _word(verdict, dev))


def rehydrate_pages(flat, pools, pages, verdict, stream=None):
    """Scatter flat into the pools' listed pages (wm_rehydrate_pages)."""
    tab, dev = _pools(pools), _device(flat)
    _need(tab.device in (None, dev) and flat.is_contiguous(), "flat is dense, on the pools' device")
    return _run("wm_rehydrate_pages", dev, stream, LIB.wm_rehydrate_pages, flat.data_ptr(),
                flat.numel() * flat.element_size(), tab.t, tab.n,
                _vec(pages, torch.int32, dev, "pages"), pages.numel(), _word(verdict, dev))
