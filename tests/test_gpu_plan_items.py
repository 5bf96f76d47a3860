"""The items that plora_attn_plan lists: every set of rows and keys once and whole, partial
rows of their own, tile items of several rounds by the length of their keys."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paged_plan_model as M  # noqa: E402
from test_gpu_paged import G, P, i32  # noqa: E402, F401

CLASSES = M.constant("kClasses")


def items(G, P, past, new, H, KH, page, group, prefix):
    """The items of few rows, those of tiles in their order, the header's words."""
    B = len(past)
    step = G.Step(B, int(np.sum(new)), page, int((np.max(past) + np.max(new)) // page) + 2)
    free = i32(np.zeros(int(sum(-(-(p + n) // page) - -(-p // page) for p, n in zip(past, new)))))
    G.kv_plan(i32(past), i32(new), free, i32([0]), i32([0]), step)
    shared = group is not None
    plan = G.AttnPlan(step, H, KH, 128, max_q=int(np.max(new)), shared=shared)
    if shared:
        segs = P.Segments(B, len(prefix))
        P.segment(i32(group), segs)
        G.attn_plan(step, plan, segs, i32(prefix))
    else:
        G.attn_plan(step, plan)
    raw = plan.plan.cpu().numpy().view(np.int32)
    head = raw[:7].tolist()
    few_cap = B + (B // 2 if shared else 0) + -(-M.FEW_TARGET // KH)
    words = lambda at, n: raw[at // 4:at // 4 + 8 * n].reshape(n, 8)
    last = words(256, few_cap)[few_cap - head[5]:]
    tile = words(256 + -(-few_cap * 32 // 256) * 256, head[1])
    return np.concatenate([words(256, head[0]), last]), tile, head


def sets(listed, few):
    """rows and keys of each set of items, which have to fill it."""
    by = {}
    for tok, row, rows, req, lo, hi, part, gathered in listed.tolist():
        by.setdefault((gathered, tok), []).append((row, rows, lo, hi, req))
    out = {}
    for k, x in by.items():
        assert len({y[4] for y in x}) == 1
        pieces = sorted({y[2:4] for y in x})
        assert all(a[1] == b[0] for a, b in zip(pieces, pieces[1:]))
        tiles = sorted({y[:2] for y in x})
        assert [t[0] for t in tiles] == list(range(0, M.TILE * len(tiles), M.TILE))
        assert all(t[1] == M.TILE for t in tiles[:-1]) and len(x) == len(tiles) * len(pieces)
        assert len(set(x)) == len(x)
        out[k] = (tiles[-1][0] + tiles[-1][1], pieces[-1][1] - pieces[0][0])
        assert (out[k][0] <= M.FEW) == few
    return out


def test_items(G, P):
    rng = np.random.default_rng(8)
    rounds = 0
    for i in range(80):
        B = int(rng.choice([1, 5, 40, 300, 700, 1100]))
        KH = int(rng.choice([1, 2, 8, 32]))
        r = int(rng.choice([1, 3, 8, 20]))
        new = rng.integers(0, int(rng.choice([2, 9, 300 if B < 50 else 20])) + 1, B)
        new[0] = max(new[0], 1)
        past = rng.integers(0, int(rng.choice([1, 500, 20000])) + 1, B)
        group, prefix = None, ()
        if rng.random() < 0.6:
            n = int(rng.integers(1, 9))
            prefix = rng.integers(0, int(rng.choice([100, 9000])), n)
            group = rng.integers(-1, n, B)
            past = past + np.where(group >= 0, prefix[group], 0)
        few, tile, head = items(G, P, past, new, KH * r, KH, 16, group, prefix)
        found, tiles = sets(few, True), sets(tile, False)
        want = M.sets_of(past, new, r, 16, group, prefix)
        assert sorted([*found.values(), *tiles.values()]) == sorted(s[:2] for s in want), i
        # partial rows
        every = np.concatenate([few, tile])
        every = every[every[:, 6] >= 0]
        at = np.concatenate([np.arange(x[6], x[6] + x[2]) for x in every]) if len(every) else []
        assert len(at) == head[2] and np.array_equal(np.sort(at), np.arange(head[2])), i
        # several rounds: by quarters of the longest piece, the longest first
        if len(tile) * KH > M.SLOTS:
            rounds += 1
            per = {k: M.cut(*s, 1, head[4])[2] for k, s in tiles.items()}
            longest = max(per.values())
            cls = [min(CLASSES - 1, (longest - per[(x[7], x[0])]) * CLASSES // longest)
                   for x in tile.tolist()]
            assert cls == sorted(cls), i
    assert rounds > 8
