"""Python binding of ``include/plora_pages.h``: upkeep of a paged cache between steps.

``kv_remap`` makes the block table of a new batch from an old one's (requests that are
continued by several, cut short, reordered or ended; their pages shared, taken and given
back), ``kv_copy`` copies the pages that it lists, and ``kv_compact`` moves the keys of
accepted paths (``tree.tree_accept``) together, each in the caches of all layers.

The calls check and forward as those of ``paged`` do.
"""
from __future__ import annotations

import ctypes

import torch

from .paged import META_WORDS, _I32, KVCache, Step, _ints, _on, _stream, plora_kv_cache, \
    plora_kv_step
from .plora import lib
from .tree import _launch

MAX_LAYERS = 1024

EXPORTED = ("plora_kv_remap_workspace_bytes", "plora_kv_remap", "plora_kv_copy",
            "plora_kv_compact")


class plora_page_pool(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("n_free", ctypes.c_int32),
                ("shares", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
                ("scratch", ctypes.c_void_p)]


class plora_kv_batch(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p)]


def _declare(L) -> None:
    P, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    CA, ST, PO, BA = (ctypes.POINTER(plora_kv_cache), ctypes.POINTER(plora_kv_step),
                      ctypes.POINTER(plora_page_pool), ctypes.POINTER(plora_kv_batch))
    L.plora_kv_remap_workspace_bytes.argtypes = [i32, i32]
    L.plora_kv_remap_workspace_bytes.restype = sz
    L.plora_kv_remap.argtypes = [BA, P, P, i32, PO, P, P, BA, P, P, P, sz, P]
    L.plora_kv_copy.argtypes = [CA, i32, P, i32, P, P]
    L.plora_kv_compact.argtypes = [CA, i32, ST, P, P, P]
    for fn in EXPORTED[1:]:
        getattr(L, fn).restype = ctypes.c_int


_declare(lib)


def kv_remap_workspace_bytes(old_batch: int, new_batch: int) -> int:
    return int(lib.plora_kv_remap_workspace_bytes(old_batch, new_batch))


class PagePool:
    """Who holds a pool's pages: shares int32 [n_pages], holders beyond the first
    (given, or zeros), and the list of free pages int32, whose head the caller keeps."""

    def __init__(self, shares, free_pages):
        self.dev = shares.get_device()
        self.shares, self.free_pages = shares, free_pages
        self.n_pages = shares.numel()
        self.scratch = torch.empty((self.n_pages, 2), dtype=_I32, device=shares.device)
        self.struct = plora_page_pool(self.n_pages, free_pages.numel(),
                                      _ints("shares", shares, _I32, 0, self.dev),
                                      _ints("free_pages", free_pages, _I32, 0, self.dev),
                                      self.scratch.data_ptr())
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, n_pages: int, device="cuda"):
        """All pages free, for a list's head of 0."""
        i32 = dict(dtype=_I32, device=device)
        return cls(torch.zeros(n_pages, **i32), torch.arange(n_pages, **i32))


class Remap:
    """The new batch of a remap from old_batch requests to new_batch: table int32
    [new_batch, max_pages] (given, or zeros), kv_len int32 [new_batch], copies int32
    [new_batch, 3], meta int32 [8], and the call's workspace."""

    def __init__(self, old_batch: int, new_batch: int, page_size: int, max_pages: int,
                 device="cuda", table=None):
        i32 = dict(dtype=_I32, device=device)
        self.old_batch, self.batch, self.page_size = old_batch, new_batch, page_size
        self.max_pages = max_pages
        self.table = table if table is not None else torch.zeros((new_batch, max_pages), **i32)
        self.kv_len = torch.zeros(new_batch, **i32)
        self.dev = self.kv_len.get_device()
        _ints("table", self.table, _I32, new_batch * max_pages, self.dev)
        if self.table.dim() > 1 and tuple(self.table.shape[1:]) != (max_pages,):
            raise ValueError("table: rows of max_pages entries expected")
        self.copies = torch.full((new_batch, 3), -1, **i32)
        self.meta = torch.zeros(META_WORDS, **i32)
        self.ws = torch.empty(kv_remap_workspace_bytes(old_batch, new_batch), dtype=torch.uint8,
                              device=device)
        self.struct = plora_kv_batch(new_batch, max_pages, self.table.data_ptr(),
                                     self.kv_len.data_ptr())
        self.ref = ctypes.byref(self.struct)
        self.out = (self.copies.data_ptr(), self.meta.data_ptr(), self.ws.data_ptr(),
                    self.ws.numel())
        self.listed = (self.copies.data_ptr(), new_batch, self.meta.data_ptr() + 4)


class Caches:
    """The caches of a model's layers, of one shape, type, strides and device."""

    def __init__(self, caches):
        self.caches = list(caches)
        if len(self.caches) > MAX_LAYERS:
            raise ValueError(f"caches: up to {MAX_LAYERS} layers expected")
        for c in self.caches:
            a, b = c.k, self.caches[0].k
            if a.shape != b.shape or a.stride() != b.stride() or a.dtype != b.dtype:
                raise ValueError("caches: layers of one shape, type and strides expected")
            _on("caches", a, self.caches[0].dev)
        self.dev = self.caches[0].dev if self.caches else -1
        self.page_size = self.caches[0].page_size if self.caches else 0
        self.n = len(self.caches)
        self.array = (plora_kv_cache * max(self.n, 1))(*(c.struct for c in self.caches))


# ---- the calls ------------------------------------------------------------------


def kv_remap(table, kv_len, src, keep, pool: PagePool, free_head, free_next, remap: Remap,
             stream=None) -> None:
    """table int32 [old_batch, max_pages], kv_len int32 [old_batch]: the old batch; src
    int32 [new_batch]: the old request that each new one continues (-1: none); keep
    int32 [new_batch] or None: how many keys of it."""
    dev, n = remap.dev, remap.old_batch
    if table.dim() != 2 or table.shape[0] < n:
        raise ValueError("table: [old_batch, max_pages] expected")
    if pool.dev != dev:
        _on("pool", pool.shares, dev)
    old = plora_kv_batch(n, table.shape[1], _ints("table", table, _I32, 0, dev),
                         _ints("kv_len", kv_len, _I32, n, dev))
    _launch("plora_kv_remap", lib.plora_kv_remap, dev, ctypes.byref(old),
            _ints("src", src, _I32, remap.batch, dev),
            None if keep is None else _ints("keep", keep, _I32, remap.batch, dev),
            remap.page_size, pool.ref, _ints("free_head", free_head, _I32, 1, dev),
            _ints("free_next", free_next, _I32, 1, dev), remap.ref, *remap.out,
            _stream(stream, dev))


def kv_copy(caches: Caches, remap: Remap, stream=None) -> None:
    """Copies the pages that the remap lists, in all layers."""
    if caches.n == 0:
        return
    dev = caches.dev
    if remap.dev != dev:
        _on("remap", remap.meta, dev)
    if remap.page_size != caches.page_size:
        raise ValueError("remap: pages of another size than the caches'")
    _launch("plora_kv_copy", lib.plora_kv_copy, dev, caches.array, caches.n, *remap.listed,
            _stream(stream, dev))


def kv_compact(caches: Caches, step: Step, path, count, stream=None) -> None:
    """path int32 [T], count int32 [batch]: as tree_accept leaves them."""
    if caches.n == 0:
        return
    dev = caches.dev
    if step.dev != dev:
        raise ValueError("step: on another device than the caches")
    _launch("plora_kv_compact", lib.plora_kv_compact, dev, caches.array, caches.n, step.ref,
            _ints("path", path, _I32, step.T, dev),
            _ints("count", count, _I32, step.batch, dev), _stream(stream, dev))
