"""Python binding of the paged key-value cache C ABI (include/hstu_cache.h): the
cache's pages and the attention of one new token over them.

Argument marshalling only: the bookkeeping, the copies and the attention run in the
HIP kernels of libhstu_jagged.so.  The functions with the C names take device
tensors; `Cache` holds a cache's tensors and workspace, `DecodePlan` the outputs and
workspace of a batch of new tokens.  Without the built library every call raises:
there is no fallback implementation.

One step of serving, for each new token of every sequence:

    start = cache.extend(slots, counts)           # room, once a step
    for each layer:
        cache.write(layer, k, v, slots, start, row_offsets, max_new, ts)
        y = plan.forward(q, u, slots, layer).y    # over the history, itself last
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional

import torch

from . import hstu

# bits of a cache's status word (include/hstu_cache.h)
HSTU_CACHE_FULL = 0x1
HSTU_CACHE_BAD_SLOT = 0x2
HSTU_CACHE_TWICE = 0x4
HSTU_CACHE_BAD_COUNT = 0x8


class CacheDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("layers", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("slots", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("ts", ctypes.c_void_p), ("tables", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("status", ctypes.c_void_p)]


class PagedOut(ctypes.Structure):
    _fields_ = [("y", ctypes.c_void_p), ("o", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_bound = False


def _lib():
    global _bound
    lib = hstu.load_library()
    if not _bound:
        P, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        C = ctypes.POINTER(CacheDesc)
        lib.hstu_cache_workspace_bytes.argtypes = [C]
        lib.hstu_cache_workspace_bytes.restype = size
        lib.hstu_cache_clear.argtypes = [C, P]
        lib.hstu_cache_extend.argtypes = [C, P, P, i32, P, P, size, P]
        lib.hstu_cache_write.argtypes = [C, i32, P, P, P, P, P, P, i32, i64, i32, P]
        lib.hstu_cache_fork.argtypes = [C, P, P, i32, P, size, P]
        lib.hstu_cache_free.argtypes = [C, P, i32, P]
        lib.hstu_cache_compact.argtypes = [C, P, P, size, P]
        lib.hstu_paged_attn_workspace_bytes.argtypes = [C, i32]
        lib.hstu_paged_attn_workspace_bytes.restype = size
        lib.hstu_paged_attn_fwd.argtypes = [P, P, C, i32, P, i32, i32, ctypes.POINTER(hstu.Rab),
                                            ctypes.POINTER(hstu.Window),
                                            ctypes.POINTER(PagedOut), P]
        for f in (lib.hstu_cache_clear, lib.hstu_cache_extend, lib.hstu_cache_write,
                  lib.hstu_cache_fork, lib.hstu_cache_free, lib.hstu_cache_compact,
                  lib.hstu_paged_attn_fwd):
            f.restype = ctypes.c_int
        _bound = True
    return lib


def _bytes(n: int) -> int:
    if n == 0:
        raise hstu.HstuError(-1, hstu.last_error())
    return n


def hstu_cache_workspace_bytes(desc: CacheDesc) -> int:
    return _bytes(_lib().hstu_cache_workspace_bytes(ctypes.byref(desc)))


def hstu_cache_clear(desc: CacheDesc, stream=None) -> None:
    hstu._check(_lib().hstu_cache_clear(ctypes.byref(desc), hstu._stream(stream)))


def hstu_cache_extend(desc: CacheDesc, slot_ids, counts, n, start, workspace,
                      stream=None) -> None:
    hstu._check(_lib().hstu_cache_extend(
        ctypes.byref(desc), hstu._ptr(slot_ids), hstu._ptr(counts), int(n), hstu._ptr(start),
        hstu._ptr(workspace), workspace.numel(), hstu._stream(stream)))


def hstu_cache_write(desc: CacheDesc, layer, k, v, timestamps, slot_ids, start, row_offsets, n,
                     total_rows, max_new, stream=None) -> None:
    hstu._check(_lib().hstu_cache_write(
        ctypes.byref(desc), int(layer), hstu._ptr(k), hstu._ptr(v), hstu._ptr(timestamps),
        hstu._ptr(slot_ids), hstu._ptr(start), hstu._ptr(row_offsets), int(n), int(total_rows),
        int(max_new), hstu._stream(stream)))


def hstu_cache_fork(desc: CacheDesc, src, dst, n, workspace, stream=None) -> None:
    hstu._check(_lib().hstu_cache_fork(
        ctypes.byref(desc), hstu._ptr(src), hstu._ptr(dst), int(n), hstu._ptr(workspace),
        workspace.numel(), hstu._stream(stream)))


def hstu_cache_free(desc: CacheDesc, slot_ids, n, stream=None) -> None:
    hstu._check(_lib().hstu_cache_free(ctypes.byref(desc), hstu._ptr(slot_ids), int(n),
                                       hstu._stream(stream)))


def hstu_cache_compact(desc: CacheDesc, live, workspace, stream=None) -> None:
    hstu._check(_lib().hstu_cache_compact(ctypes.byref(desc), hstu._ptr(live),
                                          hstu._ptr(workspace), workspace.numel(),
                                          hstu._stream(stream)))


def hstu_paged_attn_workspace_bytes(desc: CacheDesc, rows) -> int:
    return _bytes(_lib().hstu_paged_attn_workspace_bytes(ctypes.byref(desc), int(rows)))


def hstu_paged_attn_fwd(q, u, desc: CacheDesc, layer, slot_ids, rows, max_len,
                        rab: Optional[hstu.Rab], win: Optional[hstu.Window], out: PagedOut,
                        stream=None) -> None:
    hstu._check(_lib().hstu_paged_attn_fwd(
        hstu._ptr(q), hstu._ptr(u), ctypes.byref(desc), int(layer), hstu._ptr(slot_ids),
        int(rows), int(max_len), ctypes.byref(rab) if rab is not None else None,
        ctypes.byref(win) if win is not None else None, ctypes.byref(out), hstu._stream(stream)))


def _check(name, t, dtype, device, shape=None) -> None:
    """The kernels read a tensor as what it has to be: a wrong one is refused here."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the cache on {device}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


class Cache:
    """A paged cache: `layers` pools of `num_pages` pages of `page_size` tokens for
    keys and values each, and `slots` sequences of up to `max_pages` pages.

    k, v [layers][num_pages][page_size][H][d]; ts [num_pages][page_size] int64 or
    None; tables [slots][max_pages], lens [slots], refs [num_pages], status [1]
    int32: device tensors that the calls below change in stream order.
    """

    def __init__(self, num_pages, page_size, H, d, slots, max_pages, layers=1,
                 dtype=torch.bfloat16, timestamps=True, device="cuda"):
        self.num_pages, self.page_size, self.H, self.d = map(int, (num_pages, page_size, H, d))
        self.slots, self.max_pages, self.layers = int(slots), int(max_pages), int(layers)
        code = hstu.HSTU_BF16 if dtype == torch.bfloat16 else \
            hstu.HSTU_F32 if dtype == torch.float32 else None
        if code is None:
            raise ValueError(f"unsupported dtype {dtype}")
        # the sizes are checked before any memory is taken for them (the pointers
        # stand in for buffers and are not read)
        self.desc = CacheDesc(code, self.layers, self.num_pages, self.page_size, self.H, self.d,
                              self.slots, self.max_pages, *([16] * 7))
        ws = hstu_cache_workspace_bytes(self.desc)
        # "cuda" is the current device
        self.device = torch.empty(0, device=device).device
        pool = (self.layers, self.num_pages, self.page_size, self.H, self.d)
        i32 = dict(dtype=torch.int32, device=self.device)
        self.k = torch.empty(pool, dtype=dtype, device=self.device)
        self.v = torch.empty(pool, dtype=dtype, device=self.device)
        self.ts = (torch.empty(self.num_pages, self.page_size, dtype=torch.int64,
                               device=self.device) if timestamps else None)
        self.tables = torch.empty(self.slots, self.max_pages, **i32)
        self.lens = torch.empty(self.slots, **i32)
        self.refs = torch.empty(self.num_pages, **i32)
        self.status = torch.empty(1, **i32)
        self.ws = hstu._workspace(ws, self.device)
        self.desc = CacheDesc(code, self.layers, self.num_pages, self.page_size, self.H, self.d,
                              self.slots, self.max_pages, hstu._ptr(self.k), hstu._ptr(self.v),
                              hstu._ptr(self.ts), hstu._ptr(self.tables), hstu._ptr(self.lens),
                              hstu._ptr(self.refs), hstu._ptr(self.status))
        self.clear()

    def _here(self) -> None:
        """The library launches on the current device."""
        if hstu._get_device is not None and hstu._get_device() != self.device.index:
            raise ValueError(f"the cache is on {self.device}, which is not the current device")

    def _rows(self, name, t) -> int:
        self._here()
        _check(name, t, torch.int32, self.device)
        if t.dim() != 1:
            raise ValueError(f"{name} must have one dimension")
        return t.numel()

    def clear(self, stream=None) -> None:
        """Ends every sequence; all pages are free."""
        self._here()
        hstu_cache_clear(self.desc, stream)

    def extend(self, slots, counts, stream=None, start=None) -> torch.Tensor:
        """Room for counts[r] more tokens of sequence slots[r]; returns the position of
        each row's first new token (int32; -1: the row is refused, see `status`)."""
        n = self._rows("slots", slots)
        _check("counts", counts, torch.int32, self.device, (n,))
        if start is None:
            start = torch.empty(n, dtype=torch.int32, device=self.device)
        _check("start", start, torch.int32, self.device, (n,))
        hstu_cache_extend(self.desc, slots, counts, n, start, self.ws, stream)
        return start

    def write(self, layer, k, v, slots, start, row_offsets, max_new, timestamps=None,
              stream=None) -> None:
        """Rows row_offsets[r] .. row_offsets[r+1]-1 of k and v [rows][H][d] become the
        tokens from start[r] on of sequence slots[r] in `layer`; with timestamps, those
        too (once a step)."""
        n = self._rows("slots", slots)
        _check("start", start, torch.int32, self.device, (n,))
        _check("row_offsets", row_offsets, torch.int64, self.device, (n + 1,))
        total = k.shape[0]
        for name, t in (("k", k), ("v", v)):
            _check(name, t, self.k.dtype, self.device, (total, self.H, self.d))
        if timestamps is not None:
            _check("timestamps", timestamps, torch.int64, self.device, (total,))
        hstu_cache_write(self.desc, layer, k, v, timestamps, slots, start, row_offsets, n, total,
                         max_new, stream)

    def fork(self, src, dst, stream=None) -> None:
        """dst[r] becomes what src[r] was before the call, on shared pages, all rows at
        once; what dst[r] held is freed."""
        n = self._rows("src", src)
        _check("dst", dst, torch.int32, self.device, (n,))
        hstu_cache_fork(self.desc, src, dst, n, self.ws, stream)

    def free(self, slots, stream=None) -> None:
        """Ends the sequences `slots`."""
        n = self._rows("slots", slots)
        hstu_cache_free(self.desc, slots, n, stream)

    def compact(self, stream=None, live=None) -> torch.Tensor:
        """Moves the pages in use to the front of the pools; returns their number (int32
        [1] on the device)."""
        self._here()
        if live is None:
            live = torch.empty(1, dtype=torch.int32, device=self.device)
        _check("live", live, torch.int32, self.device, (1,))
        hstu_cache_compact(self.desc, live, self.ws, stream)
        return live


@dataclass
class DecodeResult:
    y: torch.Tensor         # [rows, H*d]
    o: torch.Tensor         # [rows, H, d]


class DecodePlan:
    """Outputs and workspace of the attention of `rows` new tokens over a cache,
    allocated once and reused; max_len, the bias tables and the window as for
    hstu.Plan (timestamps are the cache's)."""

    def __init__(self, cache: Cache, rows, max_len, pos_w=None, time_w=None, num_buckets=128,
                 alpha=1.0, window=None, sinks=0):
        self.cache, self.rows, self.N = cache, int(rows), int(max_len)
        H, d, dev = cache.H, cache.d, cache.device
        if pos_w is not None:
            _check("pos_w", pos_w, torch.float32, dev, (H, 2 * self.N - 1))
        if time_w is not None:
            _check("time_w", time_w, torch.float32, dev, (H, int(num_buckets)))
        self.rab = hstu.make_rab(pos_w, time_w, None, num_buckets, alpha)
        self.win = hstu.make_window(window, sinks)
        self._keep = (pos_w, time_w)
        cache._here()
        self.ws = hstu._workspace(hstu_paged_attn_workspace_bytes(cache.desc, self.rows), dev)
        self.y = torch.empty(self.rows, H * d, dtype=cache.k.dtype, device=dev)
        self.o = torch.empty(self.rows, H, d, dtype=cache.k.dtype, device=dev)
        self.out = PagedOut(hstu._ptr(self.y), hstu._ptr(self.o), hstu._ptr(self.ws),
                            self.ws.numel())

    def forward(self, q, u, slots, layer=0, stream=None) -> DecodeResult:
        """q [rows][H][d] and u [rows][H*d] of the last tokens of the sequences `slots`,
        whose own keys and values are in the cache already."""
        c = self.cache
        if c._rows("slots", slots) != self.rows:
            raise ValueError(f"{slots.numel()} slots for a plan of {self.rows} rows")
        _check("q", q, c.k.dtype, c.device, (self.rows, c.H, c.d))
        _check("u", u, c.k.dtype, c.device, (self.rows, c.H * c.d))
        hstu_paged_attn_fwd(q, u, c.desc, layer, slots, self.rows, self.N, self.rab, self.win,
                            self.out, stream)
        return DecodeResult(self.y, self.o)
