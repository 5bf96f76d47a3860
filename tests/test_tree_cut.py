"""A cut node (a parent out of range, a cut ancestor, a tree of too many nodes) is not
accepted (include/plora_tree.h), where it is one of the given ones as well: its attention
is zeros, and the target behind it and its key mean nothing."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tree as OT  # noqa: E402
from test_gpu_paged import G, i32  # noqa: E402, F401
from test_gpu_tree import R, check_accept, planned, shape_of  # noqa: E402, F401

MANY = OT.MAX_NODES + 6


def a_prompt_and_a_tree(n, prompt):
    """A chain of prompt nodes with two roots of drafts hung on its end."""
    p = np.arange(n) - 1
    p[prompt + 1:] = prompt - 1
    return p


# parent, given, the path where every node's token is 7 and so is every target
CASES = [
    ([-3, 0, 1], None, []),                      # the root itself
    ([0, 0, 1], 2, []),                          # its own parent
    ([-1, 0, 9, 2, 1, 4], 4, [0, 1, 4, 5]),      # the prompt's end: from its last fine node on
    ([-1, 0, -2, 1, 3], 4, [0, 1, 3, 4]),        # one in the middle, nothing hung on it
    ([-1, 0, -2, 2, 3], 5, [0, 1]),              # and all behind it
    ([-1, 4, 0], 2, [0, 2]),
    (a_prompt_and_a_tree(MANY, 1000), 1000, []),
    (a_prompt_and_a_tree(1024, 1000), 1000, list(range(1001))),
    (np.arange(MANY) - 1, 1000, list(range(MANY))),      # a chain of any length is not cut
]


def expected(parent, path, past):
    n = len(parent)
    return dict(path=path + [-1] * (n - len(path)), count=[len(path)],
                token=[7 if path else -1], kv_len=[past + len(path)])


@pytest.mark.parametrize("parent,given,path", CASES)
def test_oracle(parent, given, path):
    n = len(parent)
    got = OT.accept(parent, [7] * n, [7] * n, None if given is None else [given], [0, n], [30 + n],
                    [0] * n, n)
    assert got == expected(parent, path, 30)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.int32, torch.int64])
@pytest.mark.parametrize("parent,given,path", CASES)
def test_accept(G, R, parent, given, path, dt):
    n = len(parent)
    _, a = check_accept(G, R, [30], [n], parent, [7] * n, [7] * n,
                        None if given is None else [given], dt)
    for k, v in expected(parent, path, 30).items():
        assert getattr(a, k).tolist() == v, k


@pytest.mark.gpu
def test_no_cut_node_is_on_a_path(G, R):
    """Random requests with wrong parents among the given nodes: what is accepted is what
    the layout did not cut."""
    rng = np.random.default_rng(12)
    new = rng.integers(1, 300, 40)
    new[5] = 1500
    parent = np.concatenate([np.where(rng.random(n) < 0.02, 10 ** 6, np.arange(n) - 1)
                             if b % 2 else shape_of("bad", int(n), rng)
                             for b, n in enumerate(new)])
    past = rng.integers(0, 50, 40)
    step, a = check_accept(G, R, past, new, parent, *rng.integers(0, 2, (2, len(parent))),
                           rng.integers(0, 200, 40), torch.int32)
    tree = R.Tree(step)
    R.tree_plan(i32(parent), step, tree)
    first, path = tree.span[:, 0].cpu().numpy(), a.path.cpu().numpy()
    at = np.repeat(np.cumsum(new) - new, new)
    on = path >= 0
    assert on.sum() > 100 and (first[at[on] + path[on]] >= 0).all()
    assert a.count[5].item() == 0 and a.kv_len[5].item() == past[5]
