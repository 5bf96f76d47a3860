"""The plan's kernel against its model in whole numbers: items of each kind, partial rows
and keys per piece, none dropped."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paged_plan_model as M  # noqa: E402
from test_gpu_paged import G, P, i32  # noqa: E402, F401


def header(G, P, past, new, H, KH, page=16, group=None, prefix=()):
    B, T = len(past), int(np.sum(new))
    step = G.Step(B, T, page, int((np.max(past) + np.max(new)) // page) + 2)
    free = i32(np.zeros(int(sum(-(-(p + n) // page) - -(-p // page) for p, n in zip(past, new)))))
    G.kv_plan(i32(past), i32(new), free, i32([0]), i32([0]), step)
    assert step.meta.tolist()[2] == 0
    plan = G.AttnPlan(step, H, KH, 128, max_q=int(np.max(new)), shared=group is not None)
    if group is not None:
        segs = P.Segments(B, len(prefix))
        P.segment(i32(group), segs)
        G.attn_plan(step, plan, segs, i32(prefix))
    else:
        G.attn_plan(step, plan)
    words = plan.plan[:28].view(torch.int32).tolist()
    assert words[6] == 0
    return tuple(words[:6])


def test_random_steps(G, P):
    rng = np.random.default_rng(3)
    for i in range(120):
        B = int(rng.choice([1, 3, 40, 300, 600, 1100]))
        KH = int(rng.choice([1, 2, 8, 32]))
        r = int(rng.choice([1, 3, 8, 16, 20]))
        new = rng.integers(0, int(rng.choice([1, 2, 9, 300 if B < 300 else 20])) + 1, B)
        new[0] = max(new[0], 1)
        past = rng.integers(0, int(rng.choice([1, 500, 20000])) + 1, B)
        group, prefix = None, ()
        if rng.random() < 0.6:
            n = int(rng.integers(1, 9))
            prefix = rng.integers(0, int(rng.choice([100, 9000])), n)
            group = rng.integers(-1, n, B)
            past = past + np.where(group >= 0, prefix[group], 0)
        page = int(rng.choice([16, 64, 256]))
        want = M.plan(M.sets_of(past, new, r, page, group, prefix), KH)
        assert header(G, P, past, new, KH * r, KH, page, group, prefix) == want, i


@pytest.mark.parametrize("H,KH", [(1, 1), (17, 1), (129, 1), (8, 8)])
def test_steps_at_the_edges(G, P, H, KH):
    for past in (0, 511, 512, 513, 1024, 1537, 100000):
        for n in (1, 8, 17, 129):
            new, at = np.full(4, n), np.full(4, past)
            assert header(G, P, at, new, H, KH) == M.plan(M.sets_of(at, new, H // KH, 16), KH)
            group, prefix = np.array([0, 0, 1, 1]), [past, past]
            assert header(G, P, at, new, H, KH, 16, group, prefix) == \
                M.plan(M.sets_of(at, new, H // KH, 16, group, prefix), KH)
