"""Python binding of ``include/plora_paged.h``: a serving step over a paged cache.

Once a step, ``kv_plan`` lays out the batch (positions, block table entries of new
pages, cache slots) and ``attn_plan`` its attention; in every layer
``rope_append`` turns q and k and stores k and v, and ``attn_paged`` attends.  As
in ``plora``, the functions forward device pointers, strides and the caller's
stream to the C ABI and raise ``PloraError`` on a non-OK status; the classes hold
the buffers a step needs as torch tensors.  Tensors of another type, shape or device
than a call takes are refused before it (TypeError, ValueError).

``rope_turns`` gives the rotation's frequencies, scaled for long contexts where
asked; ``run_layers`` runs a step's layers as a serving loop would.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .plora import PLORA_OK, PloraError, lib, plora_segments

BF16, FP16 = 0, 1
HALF, INTERLEAVED = 0, 1
_LAYOUT = {"half": HALF, "interleaved": INTERLEAVED}
META_WORDS = 8
MAX_BATCH = 16384
MAX_TOKENS = 1 << 20
PAGE_MIN, PAGE_MAX = 16, 256
SHARE_ROWS = 128
PLAN_LEFT_OUT = 6

EXPORTED = ("plora_kv_plan", "plora_rope", "plora_rope_append", "plora_attn_plan_bytes",
            "plora_attn_paged_workspace_bytes", "plora_attn_plan", "plora_attn_paged",
            "plora_paged_last_hip_error")


class plora_kv_cache(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


class plora_kv_step(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("T", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("q_start", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("req", ctypes.c_void_p), ("slot", ctypes.c_void_p),
                ("meta", ctypes.c_void_p)]


class plora_attn_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "T", "heads", "kv_heads", "head_dim",
                                              "max_q", "shared", "reserved")]


def _declare(L) -> None:
    P, i32, i64, sz, F = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                          ctypes.c_float)
    CA, ST, SH = (ctypes.POINTER(plora_kv_cache), ctypes.POINTER(plora_kv_step),
                  ctypes.POINTER(plora_attn_shape))
    SG = ctypes.POINTER(plora_segments)
    L.plora_kv_plan.argtypes = [P, P, P, i32, P, P, ST, P]
    L.plora_rope.argtypes = [P, i64, i64, P, P, i32, i32, i32, i32, i32, F, i32, i32, P, i64,
                             i64, P]
    L.plora_rope_append.argtypes = [P, i64, i64, P, i64, i64, P, i64, i64, P, P, P, i32, i32,
                                    i32, i32, F, CA, P, i64, i64, P]
    L.plora_attn_plan.argtypes = [ST, SH, SG, P, i32, P, sz, P]
    L.plora_attn_paged.argtypes = [P, i64, i64, CA, ST, SH, F, P, sz, P, i64, i64, P, sz, P]
    for fn in ("plora_kv_plan", "plora_rope", "plora_rope_append", "plora_attn_plan",
               "plora_attn_paged"):
        getattr(L, fn).restype = ctypes.c_int
    for fn in ("plora_attn_plan_bytes", "plora_attn_paged_workspace_bytes"):
        getattr(L, fn).argtypes = [SH]
        getattr(L, fn).restype = sz
    L.plora_paged_last_hip_error.argtypes = []
    L.plora_paged_last_hip_error.restype = i32


_declare(lib)


# (int16: bf16 bits, as in plora)
_CODE = {torch.bfloat16: BF16, torch.int16: BF16, torch.float16: FP16}
_I32, _I64 = torch.int32, torch.int64
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, dev: int) -> int:
    """The stream given, or the current one of GPU dev, which all tensors of the
    call are on (-1: they are the host's, whose addresses no kernel may get)."""
    if dev < 0:
        raise ValueError("GPU tensors expected")
    if stream is not None:
        return int(stream.cuda_stream)
    if _current is not None:
        return _current(dev)
    return int(torch.cuda.current_stream(dev).cuda_stream)


def _ok(fn: str, status: int) -> None:
    if status != PLORA_OK:
        raise PloraError(fn, status, lib.plora_paged_last_hip_error)


def _dtype(t) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"bf16 or fp16 tensor expected, got {t.dtype}")
    return code


def _on(name: str, t, dev: int) -> None:
    if t.get_device() != dev:
        raise ValueError(f"{name}: on another device than the call's other tensors")


def _heads(name: str, t, dtype: int, dev: int):
    """Pointer, token stride and head stride of a [T, heads, dim] tensor on dev."""
    s = t.stride()
    if len(s) != 3 or (s[2] != 1 and t.shape[2] > 1):
        raise ValueError(f"{name}: a [T, heads, dim] tensor with contiguous dim expected")
    if _CODE.get(t.dtype) != dtype:
        raise TypeError(f"{name}: has another type than expected")
    if t.get_device() != dev:
        _on(name, t, dev)
    return t.data_ptr(), s[0], s[1]


def _ints(name: str, t, dtype, n: int, dev: int):
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of at least {n} entries expected")
    if t.get_device() != dev:
        _on(name, t, dev)
    return t.data_ptr()


class KVCache:
    """One layer's cache: k and v [n_pages, kv_heads, page_size, head_dim], of
    the same strides (any, with contiguous head_dim)."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v: 4-d tensors of one shape, type and strides expected")
        if k.shape[3] > 1 and k.stride(3) != 1:
            raise ValueError("k and v: contiguous head_dim expected")
        self.dev = k.get_device()
        _on("v", v, self.dev)
        self.k, self.v = k, v
        self.n_pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.dtype = _dtype(k)
        self.struct = plora_kv_cache(self.n_pages, self.page_size, self.kv_heads, self.head_dim,
                                     self.dtype, 0, k.data_ptr(), v.data_ptr(), k.stride(0),
                                     k.stride(1), k.stride(2))
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=None,
              device="cuda"):
        shape = (n_pages, kv_heads, page_size, head_dim)
        mk = lambda: torch.zeros(shape, dtype=dtype or torch.bfloat16, device=device)
        return cls(mk(), mk())


class Step:
    """A step's buffers (plora_kv_step): the block table (given, or zeros), and
    what kv_plan fills."""

    def __init__(self, batch: int, T: int, page_size: int, max_pages: int, device="cuda",
                 table=None):
        self.batch, self.T, self.page_size, self.max_pages = batch, T, page_size, max_pages
        i32 = dict(dtype=torch.int32, device=device)
        self.table = table if table is not None else torch.zeros((batch, max_pages), **i32)
        self.q_start = torch.zeros(batch + 1, **i32)
        self.dev = self.q_start.get_device()
        _ints("table", self.table, _I32, batch * max_pages, self.dev)
        if self.table.dim() > 1 and tuple(self.table.shape[1:]) != (max_pages,):
            raise ValueError("table: rows of max_pages entries expected")
        self.kv_len = torch.zeros(batch, **i32)
        self.pos = torch.zeros(T, **i32)
        self.req = torch.full((T,), -1, **i32)
        self.slot = torch.full((T,), -1, dtype=torch.int64, device=device)
        self.meta = torch.zeros(META_WORDS, **i32)
        self.struct = plora_kv_step(batch, T, page_size, max_pages, self.table.data_ptr(),
                                    self.q_start.data_ptr(), self.kv_len.data_ptr(),
                                    self.pos.data_ptr(), self.req.data_ptr(),
                                    self.slot.data_ptr(), self.meta.data_ptr())
        self.ref = ctypes.byref(self.struct)


class AttnPlan:
    """A step's attention plan and the workspace its layers' calls use (one at a
    time: calls that share a workspace must not overlap)."""

    def __init__(self, step: Step, heads: int, kv_heads: int, head_dim: int, max_q: int,
                 shared: bool = False, device="cuda"):
        self.shape = plora_attn_shape(step.batch, step.T, heads, kv_heads, head_dim, max_q,
                                      int(shared), 0)
        self.ref = ctypes.byref(self.shape)
        self.q_shape = (step.T, heads, head_dim)
        u8 = dict(dtype=torch.uint8, device=device)
        self.plan = torch.zeros(attn_plan_bytes(self.shape), **u8)
        self.ws = torch.empty(attn_paged_workspace_bytes(self.shape), **u8)
        self.dev = self.ws.get_device()

    @property
    def left_out(self):
        """int32 [1] on the GPU: the requests whose tokens the plan last laid out
        leaves out, their outputs zeros (more than max_q of them, say)."""
        if self.plan.numel() == 0:
            return torch.zeros(1, dtype=torch.int32, device=self.plan.device)
        return self.plan[4 * PLAN_LEFT_OUT:4 * PLAN_LEFT_OUT + 4].view(torch.int32)


def attn_plan_bytes(shape: plora_attn_shape) -> int:
    return int(lib.plora_attn_plan_bytes(ctypes.byref(shape)))


def attn_paged_workspace_bytes(shape: plora_attn_shape) -> int:
    return int(lib.plora_attn_paged_workspace_bytes(ctypes.byref(shape)))


# ---- the calls ------------------------------------------------------------------


def kv_plan(past, n_new, free_pages, free_head, free_next, step: Step, stream=None) -> None:
    """past, n_new int32 [batch]; free_pages int32, handed out from entry
    free_head[0] on; free_next[0] is the entry after."""
    n, dev = step.batch, step.dev
    _ok("plora_kv_plan", lib.plora_kv_plan(
        _ints("past", past, _I32, n, dev), _ints("n_new", n_new, _I32, n, dev),
        _ints("free_pages", free_pages, _I32, 0, dev), free_pages.numel(),
        _ints("free_head", free_head, _I32, 1, dev), _ints("free_next", free_next, _I32, 1, dev),
        step.ref, _stream(stream, dev)))


def rope(x, pos, turns, out, layout: str = "half", scale: float = 1.0, inverse: bool = False,
         stream=None) -> None:
    """x, out [T, heads, dim]; rot = 2 turns.numel() elements of each head turn;
    inverse gives the input's gradient from the output's."""
    if out.shape != x.shape:
        raise ValueError("out: x's shape expected")
    dt, dev = _dtype(x), x.get_device()
    px, xt, xh = _heads("x", x, dt, dev)
    po, ot, oh = _heads("out", out, dt, dev)
    T, H, D = x.shape
    _ok("plora_rope", lib.plora_rope(
        px, xt, xh, _ints("pos", pos, _I32, T, dev), _ints("turns", turns, _I64, 0, dev), T, H, D,
        2 * turns.numel(), _LAYOUT[layout], scale, inverse, dt, po, ot, oh, _stream(stream, dev)))


def rope_append(q, k, v, pos, slot, turns, cache: KVCache, q_out, layout: str = "half",
                scale: float = 1.0, stream=None) -> None:
    """q, q_out [T, heads, dim], k, v [T, kv_heads, dim], pos int32 [T], slot
    int64 [T]: q turned into q_out, k turned into the cache, v stored there."""
    dt, dev = cache.dtype, cache.dev
    pq, qt, qh = _heads("q", q, dt, dev)
    pk, kt, kh = _heads("k", k, dt, dev)
    pv, vt, vh = _heads("v", v, dt, dev)
    po, ot, oh = _heads("q_out", q_out, dt, dev)
    shape, kv_shape = q.shape, k.shape
    T, H, D = shape
    if D != cache.head_dim or q_out.shape != shape or kv_shape != (T, cache.kv_heads, D) or \
            v.shape != kv_shape:
        raise ValueError("q, k, v, q_out: shapes do not fit each other and the cache")
    _ok("plora_rope_append", lib.plora_rope_append(
        pq, qt, qh, pk, kt, kh, pv, vt, vh, _ints("pos", pos, _I32, T, dev),
        _ints("slot", slot, _I64, T, dev), _ints("turns", turns, _I64, 0, dev), T, H,
        2 * turns.numel(), _LAYOUT[layout], scale, cache.ref, po, ot, oh, _stream(stream, dev)))


def attn_plan(step: Step, plan: AttnPlan, segs=None, prefix_len=None, stream=None) -> None:
    """segs: the batch's groups (plora.Segments filled by plora.segment from a
    group id per request); prefix_len int32 [n_groups]."""
    groups, lens, n, dev = None, None, 0, step.dev
    _on("plan", plan.ws, dev)
    if segs is not None:
        _on("segs", segs.perm, dev)
        groups, n = ctypes.byref(segs.struct), segs.n_adapters
    if prefix_len is not None:
        lens = _ints("prefix_len", prefix_len, _I32, n, dev)
    _ok("plora_attn_plan", lib.plora_attn_plan(
        step.ref, plan.ref, groups, lens, n, plan.plan.data_ptr(), plan.plan.numel(),
        _stream(stream, dev)))


def attn_paged(q, cache: KVCache, step: Step, plan: AttnPlan, scale: float, out,
               stream=None) -> None:
    """q, out [T, heads, head_dim]."""
    dt, dev = cache.dtype, cache.dev
    pq, qt, qh = _heads("q", q, dt, dev)
    po, ot, oh = _heads("out", out, dt, dev)
    if q.shape != plan.q_shape or out.shape != plan.q_shape:
        raise ValueError("q, out: the plan's [T, heads, head_dim] expected")
    if step.dev != dev or plan.dev != dev:
        raise ValueError("step, plan: on another device than the cache")
    _ok("plora_attn_paged", lib.plora_attn_paged(
        pq, qt, qh, cache.ref, step.ref, plan.ref, scale, plan.plan.data_ptr(),
        plan.plan.numel(), po, ot, oh, plan.ws.data_ptr(), plan.ws.numel(),
        _stream(stream, dev)))


# ---- the rotation's frequencies ---------------------------------------------------


def rope_turns(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original: int = 0, low: float = 1.0, high: float = 32.0, device="cuda"):
    """Turns per position of the rot/2 pairs, in units of 2^-64, as an int64
    tensor of the bits.  Pair i turns base^(-2i/rot) radians a position.

    scaling "linear" divides every frequency by factor; "base" raises the base by
    factor^(rot/(rot-2)), so that the slowest pair is stretched by factor and the
    fastest keeps its frequency; "bands" divides by factor the pairs that make
    fewer than low turns over the original context, keeps those that make more
    than high, and blends between in proportion to the turns."""
    import numpy as np
    if rot < 0 or rot % 2 or base <= 0 or factor <= 0:
        raise ValueError("rot: even and not negative, base and factor: positive")
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    w = float(base) ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
    if scaling == "linear":
        w = w / factor
    elif scaling == "bands":
        if original <= 0 or high <= low:
            raise ValueError("bands: the original context and low < high expected")
        turns = original * w / (2 * math.pi)
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
        w = w * keep + w / factor * (1.0 - keep)
    elif scaling not in ("none", "base"):
        raise ValueError(f"scaling: {scaling!r} is not known")
    whole = [int(f * 2.0 ** 64) % 2 ** 64 for f in w / (2 * math.pi)]
    bits = np.array(whole, dtype=np.uint64).view(np.int64)
    return torch.from_numpy(bits).to(device)


# ---- a step -----------------------------------------------------------------------


def run_layers(step: Step, plan: AttnPlan, layers, turns, scale: float, layout: str = "half",
               rope_scale: float = 1.0, stream=None) -> None:
    """The layers of a planned step: for each (q, k, v, cache, out), q is turned
    in place, k and v go to the cache, out is the attention."""
    for q, k, v, cache, out in layers:
        rope_append(q, k, v, step.pos, step.slot, turns, cache, q, layout, rope_scale, stream)
        attn_paged(q, cache, step, plan, scale, out, stream)
