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
import struct

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


# The checks below are on a decoding step's way, where a call's kernel runs
# for a few microseconds: each is one expression over the tensor's cheapest
# properties (a device is its number), and words are made only for an error.


def _vec(t, dtype, dev, n, name):
    """Address of a dense tensor of at least n entries."""
    if (t.dtype is dtype and t.get_device() == dev and t.numel() >= n and t.is_contiguous()):
        return t.data_ptr()
    raise ValueError(f"{name} is a dense {dtype} tensor of at least {n} entries on device {dev}")


def _word(t, dev):
    """Address of the verdict word (None -> NULL)."""
    if t is None:
        return None
    if t.get_device() == dev and t.dtype in _WORD and t.numel() >= 1:
        return t.data_ptr()
    raise ValueError(f"verdict is a 32-bit word on device {dev}")


_WORD = (torch.int32, torch.uint32)


def _device(t) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("libwm takes device tensors")
    return dev


def _run(where, dev, stream, fn, *args):
    """fn(*args, stream) on dev: a stream belongs to a device, and a kernel is
    launched on the current one."""
    if stream is None:
        s = torch._C._cuda_getCurrentRawStream(dev)
    else:
        _need(stream.device.index == dev, f"the stream is of {stream.device}, the tensors of {dev}")
        s = stream.cuda_stream
    if dev == torch._C._cuda_getDevice():
        return _check(fn(*args, s), where)
    with torch.cuda.device(dev):
        return _check(fn(*args, s), where)


_pack_cache = struct.Struct("=8Q6I").pack
_pack_rows = struct.Struct("=3Q2I").pack


def cache_desc(k_cache, v_cache, k_scale, v_scale) -> Cache:
    """The library's description of one layer's cache."""
    dev = _device(k_cache)
    _need(k_cache.dim() == 4, "codes are [blocks, heads, .., ..]")
    n, h, bt, d = k_cache.shape
    ks, vs, fmt = k_cache.stride(), v_cache.stride(), _FORMAT.get(k_cache.dtype)
    if fmt is None or v_cache.dtype is not k_cache.dtype:
        raise ValueError("key and value codes are of one 8-bit float type")
    if v_cache.shape != (n, h, d, bt):
        raise ValueError("value codes are [blocks, heads, dim, block_tokens]")
    dense = ks[2] == d and vs[2] == bt and ks[3] == 1 and vs[3] == 1
    if not dense or (h > 1 and (ks[1] != bt * d or vs[1] != bt * d)):
        raise ValueError("a block's codes are dense")
    k_step, v_step = k_scale.stride(), v_scale.stride()
    for s, step in ((k_scale, k_step), (v_scale, v_step)):
        if s.dtype is not torch.float32 or s.shape != (n, h) or (h > 1 and step[1] != 1):
            raise ValueError("scales are float32 [blocks, heads], dense within a block")
    if not dev == v_cache.get_device() == k_scale.get_device() == v_scale.get_device():
        raise ValueError("a cache's tensors are on one device")
    one = n == 1  # the stride of a single block says nothing
    page = h * bt * d
    return Cache.from_buffer_copy(_pack_cache(
        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
        page if one else ks[0], page if one else vs[0], h if one else k_step[0],
        h if one else v_step[0], n, h, bt, d, fmt, 0))


def _rows(t, heads, dim, dev, name) -> Rows:
    dt, shape, step = _DTYPE.get(t.dtype), t.shape, t.stride()
    if (dt is None or len(shape) != 3 or shape[1] != heads or shape[2] != dim or step[2] != 1
            or t.get_device() != dev):
        raise ValueError(f"{name} is [tokens, {heads}, {dim}] of bfloat16 or float16 on device "
                         f"{dev}, its vectors dense")
    return Rows.from_buffer_copy(_pack_rows(t.data_ptr(), step[0], step[1], dt, 0))


def _table(t, n, dev):
    """(address, row stride, width) of a block table of at least n rows."""
    step = t.stride()
    if (t.dtype is not torch.int32 or len(step) != 2 or t.shape[0] < n
            or (step[1] != 1 and t.shape[1] > 1) or t.get_device() != dev):
        raise ValueError(f"block_table is int32 [requests, max_blocks] on device {dev}")
    width = t.shape[1]
    return t.data_ptr(), step[0] if t.shape[0] > 1 else width, width


def page_tables(old_len, new_len, block_tokens, block_table, free_ring, pool_in, pool_out,
                slot_map, q_start, verdict, stream=None):
    """Block tables and slot maps of a step that takes request r from
    old_len[r] to new_len[r] tokens (wm_page_tables).  block_table is
    [requests, max_blocks], free_ring the ring of free blocks, pool_in and
    pool_out {first place, count}; slot_map is int64, the rest int32."""
    dev, i32, n = _device(old_len), torch.int32, old_len.numel()
    return _run("wm_page_tables", dev, stream, LIB.wm_page_tables,
                _vec(old_len, i32, dev, n, "old_len"), _vec(new_len, i32, dev, n, "new_len"), n,
                block_tokens, *_table(block_table, n, dev),
                _vec(free_ring, i32, dev, 1, "free_ring"), free_ring.numel(),
                _vec(pool_in, i32, dev, 2, "pool_in"), _vec(pool_out, i32, dev, 2, "pool_out"),
                _vec(slot_map, torch.int64, dev, 0, "slot_map"), slot_map.numel(),
                _vec(q_start, i32, dev, n + 1, "q_start"), _word(verdict, dev))


def cache_append(k, v, k_cache, v_cache, k_scale, v_scale, slot_map, q_start, verdict=None,
                 stream=None):
    """Store new keys and values [tokens, heads, dim] where slot_map says
    (wm_cache_append); q_start has an entry per request and one more."""
    c = cache_desc(k_cache, v_cache, k_scale, v_scale)
    dev, n, h, d = k_cache.get_device(), k.shape[0], k_cache.shape[1], k_cache.shape[3]
    kr, vr = _rows(k, h, d, dev, "k"), _rows(v, h, d, dev, "v")
    if v.shape[0] != n or v.dtype is not k.dtype:
        raise ValueError("k and v have the same tokens and type")
    starts = _vec(q_start, torch.int32, dev, 1, "q_start")
    return _run("wm_cache_append", dev, stream, LIB.wm_cache_append, c, kr, vr,
                _vec(slot_map, torch.int64, dev, n, "slot_map"), starts, q_start.numel() - 1, n,
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
    dev, i32 = k_cache.get_device(), torch.int32
    n, hq, d = q.shape
    qr, outr = _rows(q, hq, k_cache.shape[3], dev, "q"), _rows(out, hq, d, dev, "out")
    if out.shape[0] != n or out.dtype is not q.dtype:
        raise ValueError("out has the tokens and type of q")
    if not (0 <= window < 1 << 31 and 0 <= max_len < 1 << 31):  # (ctypes would cut them)
        raise ValueError("window and max_len are below 2^31")
    n_req = lens.numel()
    return _run("wm_cache_attend", dev, stream, LIB.wm_cache_attend, c, qr, outr,
                None if lse is None else _vec(lse, torch.float32, dev, n * hq, "lse"), hq,
                *_table(block_table, n_req, dev), _vec(lens, i32, dev, 0, "lens"),
                _vec(q_start, i32, dev, n_req + 1, "q_start"), n_req, n, max_len, scale, window,
                _word(verdict, dev),
                None if ws is None else _vec(ws, ws.dtype, dev, 0, "ws"),
                0 if ws is None else ws.numel() * ws.element_size())


class PoolTable:
    """Host table of pools [blocks, ...] (device tensors whose pages are dense;
    the stride between pages is free); build it once to move the pages of many
    sessions."""

    def __init__(self, pools):
        self.n = len(pools)
        self.pools = list(pools)  # the table holds their addresses
        self.t = (Pool * max(self.n, 1))()
        self.device = _device(pools[0]) if self.n else None
        for i, x in enumerate(pools):
            _need(x.dim() >= 1 and x.shape[0] > 0 and x[0].is_contiguous()
                  and x.get_device() == self.device,
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
                _vec(pages, torch.int32, dev, 0, "pages"), pages.numel(), flat.data_ptr(),
                flat.numel() * flat.element_size(), _word(verdict, dev))


def rehydrate_pages(flat, pools, pages, verdict, stream=None):
    """Scatter flat into the pools' listed pages (wm_rehydrate_pages)."""
    tab, dev = _pools(pools), _device(flat)
    _need(tab.device in (None, dev) and flat.is_contiguous(), "flat is dense, on the pools' device")
    return _run("wm_rehydrate_pages", dev, stream, LIB.wm_rehydrate_pages, flat.data_ptr(),
                flat.numel() * flat.element_size(), tab.t, tab.n,
                _vec(pages, torch.int32, dev, 0, "pages"), pages.numel(), _word(verdict, dev))
