"""CPU oracle of trees of drafted tokens (include/plora_tree.h).

TEST INFRASTRUCTURE ONLY, as oracle.paged: plain loops in float64 and whole numbers,
sharing no code with the product.
"""
from __future__ import annotations

import numpy as np

MAX_NODES = 1024


def rows(q_start, req, b):
    """The rows of request b's tokens, none if the step left it out."""
    lo, hi = int(q_start[b]), int(q_start[b + 1])
    return range(lo, hi) if hi > lo and int(req[lo]) == b else range(lo, lo)


def paths(parent):
    """For every node of one request the numbers from its root to itself; None for a
    cut one."""
    n = len(parent)
    if n > MAX_NODES and any(int(p) != i - 1 for i, p in enumerate(parent)):
        return [None] * n
    out = []
    for i, p in enumerate(parent):
        p = int(p)
        if p == -1:
            out.append([i])
        elif p < -1 or p >= i or out[p] is None:
            out.append(None)
        else:
            out.append(out[p] + [i])
    return out


def tree_plan(parent, q_start, kv_len, req, T):
    B = len(kv_len)
    pos, span, info = [0] * T, [(-1, -2)] * T, [(0, 0)] * B
    for b in range(B):
        at = rows(q_start, req, b)
        par = [int(parent[t]) for t in at]
        n, way = len(par), paths(par)
        past = int(kv_len[b]) - n
        kids = {}
        for i in range(n):
            if way[i] is not None:
                kids.setdefault(par[i], []).append(i)
        number, first, last = 0, {}, {}
        stack = [(i, False) for i in reversed(kids.get(-1, []))]
        while stack:
            i, done = stack.pop()
            if done:
                last[i] = number - 1
                continue
            first[i] = number
            number += 1
            stack.append((i, True))
            stack += [(c, False) for c in reversed(kids.get(i, []))]
        for i, t in enumerate(at):
            if way[i] is not None:
                pos[t], span[t] = past + len(way[i]) - 1, (first[i], last[i])
        info[b] = (int(any(p != i - 1 for i, p in enumerate(par))), way.count(None))
    return dict(pos=pos, span=span, info=info)


def attention(q, k, v, table, q_start, kv_len, req, parent, page, scale):
    """q [T, heads, dim], k, v [pages, kv_heads, page, dim] float64.  Returns the output
    and sum_j p_j |v_j|."""
    T, H, D = q.shape
    KH = k.shape[1]
    r = H // KH
    out, size = np.zeros((T, H, D)), np.zeros((T, H, D))
    for b in range(len(kv_len)):
        at = rows(q_start, req, b)
        way = paths([int(parent[t]) for t in at])
        past = int(kv_len[b]) - len(way)
        for i, t in enumerate(at):
            if way[i] is None:
                continue
            idx = np.concatenate([np.arange(past), past + np.array(way[i], np.int64)])
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


def accept(parent, drafted, target, given, q_start, kv_len, req, T):
    B = len(kv_len)
    path, count, token, kept = [-1] * T, [], [], []
    for b in range(B):
        at = rows(q_start, req, b)
        par = [int(parent[t]) for t in at]
        n, way = len(par), paths(par)
        certain = min(max(int(given[b]) if given is not None else 1, 0), n)
        nodes = [i for i in range(certain) if way[i] is not None]
        while nodes:
            cur = nodes[-1]
            fits = [c for c in range(n) if way[c] is not None and par[c] == cur
                    and int(drafted[at[c]]) == int(target[at[cur]])]
            if not fits:
                break
            nodes.append(fits[0])
        for i, x in enumerate(nodes):
            path[at[i]] = x
        count.append(len(nodes))
        token.append(int(target[at[nodes[-1]]]) if nodes else -1)
        kept.append(int(kv_len[b]) - (n - len(nodes)))
    return dict(path=path, count=count, token=token, kv_len=kept)
