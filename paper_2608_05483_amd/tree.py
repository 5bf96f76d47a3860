"""Python binding of ``include/plora_tree.h``: trees of drafted tokens in a step over
a paged cache.

After ``paged.kv_plan``, ``tree_plan`` lays out the step's trees from each node's
parent; in every layer ``paged.rope_append`` takes the tree's positions and
``attn_tree`` the place of ``paged.attn_paged``; after the model's choice behind every
node, ``tree_accept`` finds the path that is kept.  ``pages.kv_compact`` and
``pages.kv_remap`` then move its keys together and give back the pages behind them.

The calls check and forward as those of ``paged`` do.
"""
from __future__ import annotations

import ctypes

import torch

from .paged import (_I32, _I64, AttnPlan, KVCache, Step, _heads, _ints, _on, _ok, _stream,
                    plora_attn_shape, plora_kv_cache, plora_kv_step, rope_append)
from .plora import lib

MAX_NODES = 1024

EXPORTED = ("plora_tree_plan", "plora_attn_tree", "plora_tree_accept")


class plora_tree(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("T", ctypes.c_int32), ("pos", ctypes.c_void_p),
                ("span", ctypes.c_void_p), ("info", ctypes.c_void_p)]


def _declare(L) -> None:
    P, i32, i64, sz, F = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                          ctypes.c_float)
    CA, ST, SH, TR = (ctypes.POINTER(plora_kv_cache), ctypes.POINTER(plora_kv_step),
                      ctypes.POINTER(plora_attn_shape), ctypes.POINTER(plora_tree))
    L.plora_tree_plan.argtypes = [P, ST, TR, P]
    L.plora_attn_tree.argtypes = [P, i64, i64, CA, ST, SH, TR, F, P, sz, P, i64, i64, P, sz, P]
    L.plora_tree_accept.argtypes = [P, P, P, i32, P, ST, P, P, P, P, P]
    for fn in EXPORTED:
        getattr(L, fn).restype = ctypes.c_int


_declare(lib)

_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(name: str, fn, dev: int, *args) -> None:
    """The call with GPU dev, which its tensors are on, as the current one: a launch on
    the default stream goes to the current GPU."""
    if _device() != dev:
        with torch.cuda.device(dev):
            return _ok(name, fn(*args))
    _ok(name, fn(*args))


class Tree:
    """What a step knows of its trees (plora_tree): pos int32 [T] for the rotation,
    span int32 [T, 2], info int32 [batch, 2] (1 for a tree that is no chain; its cut
    nodes)."""

    def __init__(self, step: Step, device="cuda"):
        i32 = dict(dtype=_I32, device=device)
        self.batch, self.T = step.batch, step.T
        self.pos = torch.zeros(step.T, **i32)
        self.span = torch.zeros((step.T, 2), **i32)
        self.info = torch.zeros((step.batch, 2), **i32)
        self.dev = self.pos.get_device()
        self.struct = plora_tree(step.batch, step.T, self.pos.data_ptr(), self.span.data_ptr(),
                                 self.info.data_ptr())
        self.ref = ctypes.byref(self.struct)


class Accepted:
    """What tree_accept leaves: path int32 [T], count int32 [batch], token [batch] of
    the tokens' type, kv_len int32 [batch]."""

    def __init__(self, step: Step, dtype=torch.int32, device="cuda"):
        if dtype not in (_I32, _I64):
            raise TypeError(f"dtype: int32 or int64 tokens expected, got {dtype}")
        i32 = dict(dtype=_I32, device=device)
        self.batch, self.T, self.dtype = step.batch, step.T, dtype
        self.path = torch.full((step.T,), -1, **i32)
        self.count = torch.zeros(step.batch, **i32)
        self.token = torch.full((step.batch,), -1, dtype=dtype, device=device)
        self.kv_len = torch.zeros(step.batch, **i32)
        self.dev = self.path.get_device()
        self.out = (self.path.data_ptr(), self.count.data_ptr(), self.token.data_ptr(),
                    self.kv_len.data_ptr())


def tree_plan(parent, step: Step, tree: Tree, stream=None) -> None:
    """parent int32 [T]: a node's parent by its number in its request, -1 for a root."""
    dev = step.dev
    if tree.dev != dev:
        _on("tree", tree.pos, dev)
    _launch("plora_tree_plan", lib.plora_tree_plan, dev,
            _ints("parent", parent, _I32, step.T, dev), step.ref, tree.ref, _stream(stream, dev))


def attn_tree(q, cache: KVCache, step: Step, plan: AttnPlan, tree: Tree, scale: float, out,
              stream=None) -> None:
    """q, out [T, heads, head_dim]."""
    dt, dev = cache.dtype, cache.dev
    pq, qt, qh = _heads("q", q, dt, dev)
    po, ot, oh = _heads("out", out, dt, dev)
    if q.shape != plan.q_shape or out.shape != plan.q_shape:
        raise ValueError("q, out: the plan's [T, heads, head_dim] expected")
    if step.dev != dev or plan.dev != dev or tree.dev != dev:
        raise ValueError("step, plan, tree: on another device than the cache")
    _launch("plora_attn_tree", lib.plora_attn_tree, dev, pq, qt, qh, cache.ref, step.ref, plan.ref,
            tree.ref, scale, plan.plan.data_ptr(), plan.plan.numel(), po, ot, oh,
            plan.ws.data_ptr(), plan.ws.numel(), _stream(stream, dev))


def tree_accept(parent, drafted, target, step: Step, accepted: Accepted, given=None,
                stream=None) -> None:
    """drafted, target [T], of accepted's type; given int32 [batch]: how many of a
    request's first nodes are certain (None: the first).  Cut nodes are not accepted, the
    given ones no more than others."""
    dev, dt, T = step.dev, accepted.dtype, step.T
    if accepted.dev != dev:
        _on("accepted", accepted.path, dev)
    if accepted.T != T or accepted.batch != step.batch:
        raise ValueError("accepted: made for another step")
    _launch("plora_tree_accept", lib.plora_tree_accept, dev,
            _ints("parent", parent, _I32, T, dev), _ints("drafted", drafted, dt, T, dev),
            _ints("target", target, dt, T, dev), 4 if dt is _I32 else 8,
            None if given is None else _ints("given", given, _I32, step.batch, dev), step.ref,
            *accepted.out, _stream(stream, dev))


def run_layers(step: Step, plan: AttnPlan, tree: Tree, layers, turns, scale: float,
               layout: str = "half", rope_scale: float = 1.0, stream=None) -> None:
    """The layers of a planned step with trees, as paged.run_layers: for each (q, k, v,
    cache, out), q is turned in place, k and v go to the cache, out is the attention."""
    for q, k, v, cache, out in layers:
        rope_append(q, k, v, tree.pos, step.slot, turns, cache, q, layout, rope_scale, stream)
        attn_tree(q, cache, step, plan, tree, scale, out, stream)
