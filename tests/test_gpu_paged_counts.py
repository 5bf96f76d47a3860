"""Requests that a step or its attention leaves out are counted."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import (BF, G, P, Batch, check, check_plan, i32,  # noqa: E402, F401
                            run_plan)


def test_requests_that_the_plan_leaves_out(G, P):
    """Those of more tokens than stated: alone, in a group, none, and more requests
    than the plan keeps in LDS."""
    for new, max_q in (([2, 9, 3], 4), ([2, 4, 3], 4), ([9, 0, 30], 4)):
        b = Batch(G, P, [10, 10, 10], new, 4, 2, max_q=max_q)
        assert b.plan.left_out.tolist() == [sum(n > max_q for n in new)]
        got = b.run(0.2)
        ref, size = b.ref(0.2)
        out = np.repeat(np.array(new) > max_q, new)
        ref[out], size[out] = 0, 0
        check(got, ref, size, BF, 40)
        assert (got[out] == 0).all()
    new = np.arange(1300) % 4
    group = np.arange(1300) % 3 - 1
    past = np.where(group >= 0, 40, 5)
    b = Batch(G, P, past, new, 2, 1, 64, group=group, prefix=[32, 32], max_q=2)
    assert b.plan.left_out.tolist() == [325]
    # a plan without the limit leaves none out, in the same buffer
    c = G.AttnPlan(b.step, 2, 1, 64, max_q=3)
    for _ in range(2):
        G.attn_plan(b.step, c)
        assert c.left_out.tolist() == [0]


def test_each_is_counted_where_it_is_left_out(G, P):
    """A request without pages by kv_plan, one of too many tokens by attn_plan."""
    table = np.arange(12).reshape(3, 4)
    step = G.Step(3, 60, 16, 4, table=i32(table))
    G.kv_plan(i32([10, 16, 20]), i32([20, 30, 1]), i32([11]), i32([0]), i32([0]), step)
    assert step.meta.tolist()[:3] == [51, 1, 1]
    plan = G.AttnPlan(step, 4, 2, 64, max_q=10)
    G.attn_plan(step, plan)
    assert plan.left_out.tolist() == [1]


def test_an_empty_plan_leaves_none_out(G, P):
    step = G.Step(0, 0, 16, 4)
    plan = G.AttnPlan(step, 4, 2, 64, max_q=1)
    G.attn_plan(step, plan)
    assert plan.left_out.tolist() == [0]


def test_requests_of_no_tokens_behind_too_many(G, P):
    """Tokens that pass the step's rows are left out with their requests; a request
    that brings none keeps its length and is not one of them, in the first chunk of
    requests and in a later one."""
    for n in (4, 1100):
        past, new = np.full(n, 16), np.zeros(n, int)
        new[1] = 30
        got, _ = run_plan(G, past, new, np.arange(9), 0, np.zeros((n, 4), int), 16, 20)
        assert list(got["meta"][:3]) == [20, 0, 1]
        assert (got["kv_len"] == 16).all() and (got["req"] == -1).all()
        assert list(got["q_start"]) == [0, 0] + [20] * (n - 1)
        check_plan(G, past, new, np.arange(9), 0, np.zeros((n, 4), int), 16, 20)


def test_no_groups_yet(G, P):
    """A batch grouped over no groups at all: every request by itself."""
    b = Batch(G, P, [10, 300, 0], [1, 1, 4], 4, 2, group=np.full(3, -1), prefix=[0])
    segs = P.Segments(3, 0)
    P.segment(i32([-1] * 3), segs)
    G.attn_plan(b.step, b.plan, segs, i32([]))
    check(b.run(0.2), *b.ref(0.2), BF, 320)
