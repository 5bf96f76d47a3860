"""The largest trees, prompts with drafts behind them, scales of any sign, and infinities
and NaN that some nodes see and others do not, in caches cut into pieces and behind shared
prefixes."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import BF, HF, G, P, check, i32  # noqa: E402, F401
from test_gpu_paged_nonfinite import check_kinds, spoil  # noqa: E402
from test_gpu_tree import R, TreeBatch, check_accept, check_tree, shape_of  # noqa: E402, F401


def behind_a_prompt(kind, n, prompt, rng):
    """A chain of prompt nodes, then a tree whose roots hang on its end."""
    p = np.arange(n) - 1
    t = shape_of(kind, n - prompt, rng)
    p[prompt:] = np.where(t >= 0, t + prompt, prompt - 1)
    return p


@pytest.mark.parametrize("kind", ["levels", "comb", "any", "star", "bad"])
@pytest.mark.parametrize("n,prompt", [(1024, 950), (1000, 999), (700, 3), (65, 64)])
def test_drafts_behind_a_prompt(G, R, kind, n, prompt):
    rng = np.random.default_rng(n)
    parent = np.concatenate([behind_a_prompt(kind, n, prompt, rng), [-1, 0], [3] * 2])
    check_tree(G, R, [77, 0], [n, 2], parent, pad=2)
    tok = rng.integers(0, 2, (2, n + 4))
    check_accept(G, R, [77, 0], [n, 2], parent, *tok, [prompt, 1], torch.int32, pad=2)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("kind", ["levels", "any", "prompt"])
def test_largest_trees(G, P, R, dt, D, kind):
    b = TreeBatch(G, P, R, [130, 9], [1024, 40], 2, 1, D, dt=dt, seed=3,
                  kinds=("levels" if kind == "prompt" else kind,))
    if kind == "prompt":
        b.parent[:1024] = behind_a_prompt("any", 1024, 950, np.random.default_rng(0))
        R.tree_plan(i32(b.parent), b.step, b.tree)
    check(b.run(0.1), *b.ref(0.1), dt, 1200)


@pytest.mark.parametrize("scale", [-0.3, 0.0, -1e-3, 3.0])
@pytest.mark.parametrize("new,H,KH", [(6, 2, 1), (40, 4, 2)])
def test_scales(G, P, R, scale, new, H, KH):
    b = TreeBatch(G, P, R, [50, 0, 700], [new, 3, new], H, KH, seed=new)
    check(b.run(scale), *b.ref(scale), BF, 800)


WHAT = [(w, v) for w in ("key", "key element", "value") for v in (math.nan, math.inf, -math.inf)]


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("what,value", WHAT)
@pytest.mark.parametrize("H,KH,new", [(2, 2, 10), (2, 1, 40)])
def test_nodes_that_are_spoilt_in_pieces(G, P, R, dt, D, what, value, H, KH, new):
    """An inner node, which its descendants see, in caches that are cut inside a tree; and
    a cached key, which all see, of another request."""
    past = [3590 - min(new, 10), 3600 - new // 2, 900]
    b = TreeBatch(G, P, R, past, [new] * 3, H, KH, D, dt=dt, seed=new)
    assert b.header()[2] > 0
    spoil(b, 0, past[0] + 1, what, value)
    spoil(b, 1, past[1] + new // 2, what, value)
    spoil(b, 2, 5, what, value)
    got = check_kinds(b, dt, 4000)
    assert np.isfinite(got[0]).all()            # (the first root sees none of them)


@pytest.mark.parametrize("what,value", WHAT)
@pytest.mark.parametrize("new,H,KH", [([2, 7, 3], 2, 1), ([9, 16, 5, 1], 8, 1)])
def test_spoilt_behind_a_shared_prefix(G, P, R, what, value, new, H, KH):
    B = len(new)
    past = 300 + np.arange(B)
    for key in (40, int(past[1])):              # of the prefix, and the second one's root
        b = TreeBatch(G, P, R, past, new, H, KH, group=[0] * B, prefix=[256], seed=key,
                      kinds=("roots",))
        spoil(b, 1, key, what, value)
        got = check_kinds(b, BF, 400)
        hit = ~np.isfinite(got).all((1, 2))
        if what == "value":
            assert hit.all() if key < 256 else hit.tolist().index(True) == new[0]
        if key >= 256:
            assert hit.sum() <= 1
