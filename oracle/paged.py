"""CPU oracle of a serving step over a paged cache (include/plora_paged.h).

TEST INFRASTRUCTURE ONLY, as oracle.attention: plain loops in float64 and whole
numbers, sharing no code with the product.
"""
from __future__ import annotations

import math

import numpy as np


def kv_plan(past, new, free, head, table, page, T):
    """The step's layout as the header words it; table is written in place.
    Returns a dict of the outputs."""
    B, max_pages = table.shape
    q_start, kv_len, pos, req, slot = [], [], [0] * T, [-1] * T, [-1] * T
    at, want, taken, out = 0, 0, 0, 0
    avail = 0 if head < 0 else len(free) - head
    for b in range(B):
        p, n = int(past[b]), int(new[b])
        q_start.append(min(at, T))
        start = at
        at = min(at + max(n, 0), T + 1)
        ok = p >= 0 and n >= 0 and p + n <= max_pages * page and (at <= T or n == 0)
        need = -(-(p + n) // page) - -(-p // page) if ok else 0
        if ok and need > 0:
            ok = want + need <= avail
            want += need
            if ok:
                taken = want
        kv_len.append(p + n if ok else max(p, 0))
        if not ok:
            out += 1
            continue
        held = -(-p // page)
        for j in range(need):
            table[b, held + j] = free[head + want - need + j]
        for i in range(n):
            t = start + i
            pos[t], req[t] = p + i, b
            e = int(table[b, (p + i) // page])
            slot[t] = -1 if e < 0 else e * page + (p + i) % page
    q_start.append(min(at, T))
    return dict(q_start=q_start, kv_len=kv_len, pos=pos, req=req, slot=slot, next=head + taken,
                meta=[min(at, T), taken, out, 0, 0, 0, 0, 0])


def rotate(x, pos, turns, layout, scale=1.0, inverse=False):
    """x [T, heads, dim] float64; turns: rot/2 whole numbers of 2^-64 turns."""
    y = np.array(x, np.float64)
    half = len(turns)
    for t in range(x.shape[0]):
        for i in range(half):
            f = 2 * math.pi * ((int(pos[t]) * int(turns[i])) % 2 ** 64 / 2.0 ** 64)
            c, s = math.cos(f), math.sin(f) * (-1 if inverse else 1)
            a, b = (i, half + i) if layout == "half" else (2 * i, 2 * i + 1)
            y[t, :, a] = scale * (x[t, :, a] * c - x[t, :, b] * s)
            y[t, :, b] = scale * (x[t, :, a] * s + x[t, :, b] * c)
    return y


def attention(q, k, v, table, q_start, kv_len, req, pos, page, scale):
    """q [T, heads, dim], k, v [pages, kv_heads, page, dim] float64.  Returns the
    output and sum_j p_j |v_j|, the size that roundings of the weights act on."""
    T, H, D = q.shape
    KH = k.shape[1]
    r = H // KH
    out, size = np.zeros((T, H, D)), np.zeros((T, H, D))
    for t in range(T):
        b = int(req[t])
        if b < 0:
            continue
        n = int(pos[t]) + 1
        idx = np.arange(n)
        pages, off = table[b][idx // page], idx % page
        for h in range(KH):
            K, V = k[pages, h, off], v[pages, h, off]
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (q[t, h * r:(h + 1) * r] @ K.T)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[t, h * r:(h + 1) * r] = p @ V
                size[t, h * r:(h + 1) * r] = p @ np.abs(V)
    return out, size
