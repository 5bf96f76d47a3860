"""Trees of drafted tokens on the GPU (include/plora_tree.h) against the oracle: the
trees' layout and the accepted paths bit for bit, attention over its row counts, cuts,
groups, masks and odd values."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tree as OT  # noqa: E402
from test_gpu_paged import BF, HF, Batch, G, P, check, f64, i32  # noqa: E402, F401

I64 = torch.int64


@pytest.fixture(scope="module")
def R():
    from paper_2608_05483_amd import tree
    return tree


def shape_of(kind, n, rng):
    """Parents of a tree of n nodes."""
    i = np.arange(n)
    if kind == "chain":
        return i - 1
    if kind == "star":
        return np.where(i == 0, -1, 0)
    if kind == "roots":
        return np.full(n, -1)
    if kind == "levels":                     # parents in rising order, as drafts have them
        return np.where(i == 0, -1, np.minimum(i - 1, np.sort(rng.integers(0, n, n)) // 2))
    if kind == "comb":                       # a long path with a leaf at every node
        return np.where(i == 0, -1, np.where(i % 2 == 1, i - 1, i - 2))
    p = np.array([rng.integers(-1, j) if j else -1 for j in i])   # any order, several roots
    if kind == "bad":                        # parents out of range here and there
        wrong = rng.random(n) < 0.2
        return np.where(wrong, rng.choice([-2, 10 ** 6, 2 ** 31 - 1, -2 ** 31], n),
                        np.where(rng.random(n) < 0.1, i + rng.integers(0, 3, n), p))
    return p


def planned(G, past, new, page=16, pad=0, T=None):
    B = len(past)
    kv = np.asarray(past) + np.asarray(new)
    max_pages = int(-(-kv.max() // page)) + 1
    need = int((-(-kv // page)).sum())
    T = int(np.sum(new)) + pad if T is None else T
    table = np.arange(B * max_pages).reshape(B, max_pages)
    step = G.Step(B, T, page, max_pages, table=i32(table))
    G.kv_plan(i32(past), i32(new), i32(np.arange(need) + 10 ** 5), i32([0]), i32([0]), step)
    return step


def host(step):
    return {k: getattr(step, k).cpu().numpy() for k in ("q_start", "kv_len", "req")}


def check_tree(G, R, past, new, parent, pad=0, T=None):
    step = planned(G, past, new, pad=pad, T=T)
    tree = R.Tree(step)
    for t in (tree.pos, tree.span, tree.info):
        t.fill_(-77)
    R.tree_plan(i32(parent), step, tree)
    torch.cuda.synchronize()
    s = host(step)
    ref = OT.tree_plan(parent, s["q_start"], s["kv_len"], s["req"], step.T)
    assert np.array_equal(tree.pos.cpu().numpy(), ref["pos"])
    assert np.array_equal(tree.span.cpu().numpy(), np.array(ref["span"]).reshape(-1, 2))
    assert np.array_equal(tree.info.cpu().numpy(), np.array(ref["info"]).reshape(-1, 2))
    return step, tree


# ---- the trees' layout ----------------------------------------------------------------


@pytest.mark.parametrize("kind", ["chain", "star", "roots", "levels", "comb", "any", "bad"])
@pytest.mark.parametrize("sizes", [[1], [2, 1, 3], [64, 65, 63], [255, 256, 257], [1023, 1024],
                                   [1025, 7]])
def test_layout(G, R, kind, sizes):
    rng = np.random.default_rng(sum(sizes))
    parent = np.concatenate([shape_of(kind, n, rng) for n in sizes] + [[5] * 3])
    check_tree(G, R, [3 * i for i in range(len(sizes))], sizes, parent, pad=3)


def test_layout_of_mixed_batches(G, R):
    rng = np.random.default_rng(8)
    kinds = ["chain", "star", "levels", "any", "bad", "comb"]
    new = np.where(rng.random(300) < 0.1, 0, rng.integers(1, 50, 300))
    new[7], new[8] = 3000, 1030                # a prompt, and a tree of too many nodes
    pick = [kinds[rng.integers(6)] for _ in range(300)]
    pick[7], pick[8] = "chain", "levels"
    parent = np.concatenate([shape_of(k, int(n), rng) for k, n in zip(pick, new)])
    check_tree(G, R, rng.integers(0, 500, 300), new, parent)


def test_layout_of_requests_left_out(G, R):
    """Negative lengths, tokens that pass T, and a batch without any."""
    parent = np.concatenate([np.arange(5) - 1, np.zeros(7), np.arange(9) - 1]).astype(int)
    check_tree(G, R, [4, -1, 30], [5, 7, 9], parent)
    check_tree(G, R, [4, 2, 30], [5, 7, 9], parent, T=15)
    check_tree(G, R, [4, 2], [0, 0], np.full(4, -1), T=4)
    step = G.Step(3, 0, 16, 4)
    G.kv_plan(i32([1, 2, 3]), i32([0] * 3), i32([]), i32([0]), i32([0]), step)
    tree = R.Tree(step)
    tree.info.fill_(5)
    R.tree_plan(i32([]), step, tree)
    assert (tree.info.cpu() == 0).all()


# ---- attention ------------------------------------------------------------------------


class TreeBatch(Batch):
    """A planned step of trees."""

    def __init__(self, G, P, R, past, new, H, KH, D=128, kinds=("levels", "any"), seed=0, **kw):
        super().__init__(G, P, past, new, H, KH, D, seed=seed, **kw)
        rng = np.random.default_rng(seed + 1)
        par = [shape_of(kinds[b % len(kinds)], int(n), rng) for b, n in enumerate(new)]
        self.parent = np.concatenate(par + [np.full(kw.get("pad", 0), -1)]).astype(np.int64)
        self.R, self.tree = R, R.Tree(self.step)
        R.tree_plan(i32(self.parent), self.step, self.tree)

    def run(self, scale):
        self.R.attn_tree(self.q, self.cache, self.step, self.plan, self.tree, scale, self.out)
        torch.cuda.synchronize()
        return f64(self.out)

    def ref(self, scale):
        s = self.step
        return OT.attention(f64(self.q), f64(self.cache.k), f64(self.cache.v),
                            s.table.cpu().numpy(), **host(s), parent=self.parent,
                            page=self.page, scale=scale)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 128), (BF, 64), (HF, 64)])
@pytest.mark.parametrize("H,KH", [(4, 4), (8, 1), (6, 2), (20, 1)])
def test_small_trees(G, P, R, dt, D, H, KH):
    """1 to 16 nodes: up to 16 rows a key head and more."""
    past, new = [0, 1, 15, 16, 37, 127, 300, 511, 0], [1, 2, 3, 5, 8, 13, 16, 7, 11]
    b = TreeBatch(G, P, R, past, new, H, KH, D, dt=dt, seed=H + D)
    check(b.run(D ** -0.5), *b.ref(D ** -0.5), dt, 600)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("kinds", [("levels",), ("star",), ("roots",), ("comb",), ("any",),
                                   ("bad",), ("chain", "levels")])
def test_kinds_of_trees(G, P, R, dt, D, kinds):
    past, new = [0, 70, 33, 500], [40, 64, 100, 7]
    b = TreeBatch(G, P, R, past, new, 4, 2, D, kinds=kinds, dt=dt, page=32, pad=5)
    got = b.run(0.11)
    check(got, *b.ref(0.11), dt, 700)
    assert (got[-5:] == 0).all()
    cut = b.tree.span[:, 0].cpu().numpy() < 0
    assert (got[cut] == 0).all() and cut[:-5].any() == (kinds == ("bad",))


@pytest.mark.parametrize("H,KH,new", [(2, 2, 10), (1, 1, 16), (2, 1, 40), (1, 1, 300),
                                      (2, 1, 700)])
def test_long_caches_cut_inside_a_tree(G, P, R, H, KH, new):
    """Few rows over many keys: pieces, some of which begin behind the last cached key,
    so that rows see none of their keys."""
    past = [3590 - min(new, 10), 3600 - new // 2, 1100, 0] if new < 300 else [900, 310, 0, 40]
    b = TreeBatch(G, P, R, past, [new] * 4, H, KH, seed=new)
    head = b.header()
    assert head[2] > 0                          # partial rows
    keys = head[3] if new * (H // KH) <= 16 else head[4]
    check(b.run(0.09), *b.ref(0.09), BF, 4000)
    assert keys < 4000


def test_a_piece_that_no_row_sees(G, P, R):
    """The last piece holds the end of the tree alone, which its first nodes and most
    of its last ones do not see."""
    for past, new in (([3580], 10), ([3576], 12)):
        b = TreeBatch(G, P, R, past, [new], 1, 1, kinds=("star",), seed=past[0])
        items = b.plan.plan[256:256 + 32 * 16].view(torch.int32).view(-1, 8).cpu().numpy()
        lo = items[:b.header()[0], 4]
        assert (lo >= past[0]).any()
        check(b.run(0.2), *b.ref(0.2), BF, 4000)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("H,KH,hi", [(2, 2, 5), (8, 1, 9), (4, 1, 40)])
def test_trees_behind_shared_prefixes(G, P, R, dt, D, H, KH, hi):
    rng = np.random.default_rng(H + hi)
    B = 20
    group = rng.choice([-1, 0, 1, 2], B)
    prefix = np.array([200, 7, 1025])
    past = rng.integers(0, 90, B) + np.where(group >= 0, prefix[group], 0)
    new = rng.integers(1, hi + 1, B)
    new[4] = 0
    b = TreeBatch(G, P, R, past, new, H, KH, D, dt=dt, group=group, prefix=prefix, seed=hi,
                  kinds=("levels", "any", "bad", "chain"))
    check(b.run(0.1), *b.ref(0.1), dt, 1200)
    c = G.AttnPlan(b.step, H, KH, D, max_q=int(new.max()))
    G.attn_plan(b.step, c)
    b.plan = c
    check(b.run(0.1), *b.ref(0.1), dt, 1200)


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("order", ["head", "key"])
def test_pages_and_orders(G, P, R, page, order):
    b = TreeBatch(G, P, R, [0, 250, 17], [33, 30, 5], 4, 2, page=page, order=order)
    check(b.run(0.2), *b.ref(0.2), BF, 300)


@pytest.mark.parametrize("D", [128, 64])
def test_chains_are_causal(G, P, R, D):
    """A batch of prompts and single tokens gives the bits of attn_paged; a tree that
    only looks like none (one node's parent is another) does not."""
    b = TreeBatch(G, P, R, [0, 700, 3], [300, 1, 70], 4, 2, D, kinds=("chain",))
    G.attn_paged(b.q, b.cache, b.step, b.plan, 0.1, b.out)
    torch.cuda.synchronize()
    want = f64(b.out)
    b.out.fill_(3)
    assert np.array_equal(b.run(0.1), want)


@pytest.mark.parametrize("H,KH,new", [(2, 1, 7), (4, 1, 50)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_nodes_of_other_branches_have_no_part(G, P, R, H, KH, new, value):
    """Infinities and NaN in the keys and values of one leaf, and behind the last
    key: only the leaf's own row is touched."""
    past = [20, 100]
    b = TreeBatch(G, P, R, past, [new, new], H, KH, kinds=("star",))
    ref, size = b.ref(0.3)
    slot, leaves = b.step.slot.cpu().numpy(), [2, new + 4]
    for t in leaves:
        p, o = divmod(int(slot[t]), 16)
        b.cache.k[p, :, o] = value
        b.cache.v[p, :, o] = value
    table = b.step.table.cpu().numpy()
    for r in range(2):
        n = past[r] + new
        if n % 16:
            b.cache.k[table[r, n // 16], :, n % 16:] = value
            b.cache.v[table[r, n // 16], :, n % 16:] = value
    got = b.run(0.3)
    rest = [t for t in range(2 * new) if t not in leaves]
    check(got[rest], ref[rest], size[rest], BF, 200)
    assert not np.isfinite(got[leaves]).all()


@pytest.mark.parametrize("new", [3, 40])
def test_scores_of_minus_infinity(G, P, R, new):
    """A node whose every seen key scores minus infinity is 0 / 0, and nobody else."""
    b = TreeBatch(G, P, R, [0], [new], 1, 1, kinds=("roots",))
    ref, size = b.ref(0.5)
    p, o = divmod(int(b.step.slot[1]), 16)
    b.q[1].fill_(1.0)
    b.cache.k[p, 0, o].fill_(-math.inf)
    got = b.run(0.5)
    assert np.isnan(got[1]).all()
    rest = [t for t in range(new) if t != 1]
    check(got[rest], ref[rest], size[rest], BF, 50)


def test_masked_and_left_out(G, P, R):
    """More tokens than the shape states, no tokens, padding."""
    b = TreeBatch(G, P, R, [10, 10, 10, 10], [2, 9, 0, 3], 4, 2, max_q=4, pad=2)
    got = b.run(0.2)
    ref, size = b.ref(0.2)
    ref[2:11], size[2:11] = 0, 0
    check(got, ref, size, BF, 20)
    assert (got[2:11] == 0).all() and (got[-2:] == 0).all()


def test_strided_on_another_stream(G, P, R):
    b = TreeBatch(G, P, R, [50, 700, 3], [1, 4, 30], 4, 2)
    want = b.run(0.1)
    T = b.q.shape[0]
    wide_q = torch.full((T, 6, 160), 3.0, dtype=BF, device="cuda")
    wide_o = torch.full((T, 6, 160), 5.0, dtype=BF, device="cuda")
    q, out = wide_q[:, 1:5, 16:144], wide_o[:, 1:5, 16:144]
    q.copy_(b.q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        R.attn_tree(q, b.cache, b.step, b.plan, b.tree, 0.1, out, stream=s)
        s.synchronize()
        assert np.array_equal(f64(out), want)
    keep = wide_o.clone()
    keep[:, 1:5, 16:144] = 5.0
    assert (keep == 5.0).all()


# ---- acceptance -----------------------------------------------------------------------


def check_accept(G, R, past, new, parent, drafted, target, given, dt, pad=0, T=None):
    step = planned(G, past, new, pad=pad, T=T)
    a = R.Accepted(step, dtype=dt)
    for t in (a.path, a.count, a.token, a.kv_len):
        t.fill_(-77)
    dev = lambda x: torch.from_numpy(np.asarray(x)).to("cuda", dt)
    R.tree_accept(i32(parent), dev(drafted), dev(target), step, a,
                  None if given is None else i32(given))
    torch.cuda.synchronize()
    ref = OT.accept(parent, drafted, target, given, **host(step), T=step.T)
    for k, v in ref.items():
        assert np.array_equal(getattr(a, k).cpu().numpy(), v), k
    return step, a


@pytest.mark.parametrize("dt", [torch.int32, I64])
@pytest.mark.parametrize("kind", ["chain", "star", "levels", "any", "bad", "comb", "roots"])
@pytest.mark.parametrize("sizes", [[1], [30, 1, 64, 65, 2], [200, 256, 257, 300], [1024],
                                   [1100, 3]])
def test_accept(G, R, dt, kind, sizes):
    """Few different tokens, so that paths are long and several children fit."""
    rng = np.random.default_rng(sum(sizes) + len(kind))
    parent = np.concatenate([shape_of(kind, n, rng) for n in sizes] + [[-1] * 2])
    T = len(parent)
    for vocab in (1, 2, 3):
        big = 0 if dt == torch.int32 else 2 ** 40
        drafted, target = big + rng.integers(0, vocab, T), big + rng.integers(0, vocab, T)
        for given in (None, rng.integers(-1, 4, len(sizes)), np.array(sizes) + 1):
            check_accept(G, R, [5] * len(sizes), sizes, parent, drafted, target, given, dt, pad=2)


def test_accept_tells_tokens_apart_by_all_their_bits(G, R):
    step, a = check_accept(G, R, [0], [3], [-1, 0, 0], [0, 1 + 2 ** 32, 1], [1, 5, 6], None, I64)
    assert a.path.tolist() == [0, 2, -1] and a.token.tolist() == [6]


def test_accept_of_requests_left_out(G, R):
    rng = np.random.default_rng(4)
    parent = np.concatenate([np.arange(5) - 1, np.zeros(7), np.arange(9) - 1]).astype(int)
    tok = rng.integers(0, 2, 21), rng.integers(0, 2, 21)
    check_accept(G, R, [4, -1, 30], [5, 7, 9], parent, *tok, None, torch.int32)
    check_accept(G, R, [4, 2, 30], [5, 7, 9], parent, *tok, None, torch.int32, T=15)
    check_accept(G, R, [4, 2], [0, 0], np.full(4, -1), tok[0][:4], tok[1][:4], None,
                 torch.int32, T=4)
    check_accept(G, R, [4, 2], [0, 0], np.full(0, -1), tok[0][:0], tok[1][:0], [1, 1],
                 torch.int32)


def test_accept_of_many_requests(G, R):
    rng = np.random.default_rng(6)
    new = rng.integers(0, 40, 700)
    new[3] = 2500
    parent = np.concatenate([shape_of("chain" if b % 5 == 3 else "levels", int(n), rng)
                             for b, n in enumerate(new)])
    tok = rng.integers(0, 3, len(parent)), rng.integers(0, 3, len(parent))
    given = np.where(np.arange(700) % 5 == 3, new, 1)
    check_accept(G, R, rng.integers(0, 99, 700), new, parent, *tok, given, torch.int32)
