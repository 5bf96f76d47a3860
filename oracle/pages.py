"""CPU oracle of the cache's upkeep (include/plora_pages.h).

TEST INFRASTRUCTURE ONLY, as oracle.paged: plain loops over whole numbers, one request
and one page after the other, sharing no code with the product.
"""
from __future__ import annotations

import numpy as np


def remap(table, kv_len, src, keep, page, shares, free, head, new_table):
    """As the header words it; shares, free and new_table are written in place.
    Returns a dict of the other outputs."""
    B, most = table.shape
    N, new_most = new_table.shape
    P = len(shares)
    clamp = lambda n, m: min(max(int(n), 0), m * page)
    held = [clamp(n, most) for n in kv_len]
    lens, wanted = [], []
    for i in range(N):
        b = int(src[i])
        n = clamp(held[b], new_most) if 0 <= b < B else 0
        if keep is not None:
            n = min(n, max(int(keep[i]), 0))
        lens.append(n)
        names = [int(table[b, j]) for j in range(-(-n // page))]
        new_table[i, :len(names)] = names
        for p in names:
            if 0 <= p < P:
                shares[p] += 1
    dropped = [int(table[b, j]) for b in range(B) for j in range(-(-held[b] // page))]
    for p in dropped:
        if 0 <= p < P:
            shares[p] -= 1
    gone = []
    for p in dropped:
        if 0 <= p < P and shares[p] < 0:
            shares[p] = 0
            gone.append(p)
    list_ok = 0 <= head <= len(free)
    put = min(len(gone), head) if list_ok else 0
    top = head - put
    if put:
        free[top:head] = gone[len(gone) - put:]
    avail = len(free) - top if list_ok else 0
    copies, short = [], 0
    for i in range(N):
        if lens[i] % page == 0:
            continue
        j = lens[i] // page
        p = int(new_table[i, j])
        if not 0 <= p < P or shares[p] == 0:
            continue
        shares[p] -= 1
        if len(copies) < avail:
            fresh = int(free[top + len(copies)])
            copies.append((p, fresh, lens[i] % page))
            new_table[i, j] = fresh
        else:
            lens[i] = j * page
            short += 1
    meta = [put, len(copies), short, len(gone) - put, 0, 0, 0, 0]
    copies_out = np.full((N, 3), -1)
    if copies:
        copies_out[:len(copies)] = copies
    return dict(kv_len=lens, copies=copies_out, meta=meta, next=top + len(copies))


def copy(pool, copies, n):
    """pool [pages, heads, page, dim] written in place."""
    P, _, page, _ = pool.shape
    for a, b, keys in copies[:n]:
        if 0 <= a < P and 0 <= b < P:
            m = min(int(keys), page)
            if m > 0:
                pool[b, :, :m] = pool[a, :, :m]


def compact(pool, q_start, req, slot, path, count):
    """pool [pages, heads, page, dim] written in place, a move after the other."""
    P, _, page, _ = pool.shape
    there = lambda s: 0 <= s < P * page
    for b in range(len(count)):
        lo, n = int(q_start[b]), int(q_start[b + 1]) - int(q_start[b])
        if n <= 0 or int(req[lo]) != b:
            continue
        for i in range(min(int(count[b]), n)):
            j = int(path[lo + i])
            if not 0 <= j < n:
                continue
            x, y = int(slot[lo + j]), int(slot[lo + i])
            if there(x) and there(y):
                pool[y // page, :, y % page] = pool[x // page, :, x % page]
