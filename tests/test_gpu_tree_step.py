"""A whole step with trees (layout, trees, attention's plan, layers, acceptance, keys
moved together, requests cut to what they keep) captured and replayed with other
requests, and on a stream of the caller's; one host tensor among a call's GPU tensors."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import BF, G, P, i32  # noqa: E402, F401
from test_gpu_pages import K  # noqa: E402, F401
from test_gpu_tree import R, shape_of  # noqa: E402, F401

I32, I64 = torch.int32, torch.int64


class Step:
    """Buffers of a step of B requests with up to n nodes each, 2 layers, behind two
    adapters' prompts."""

    def __init__(self, G, P, R, K, B=6, n=20, page=16, H=8, KH=2, D=64):
        g = torch.Generator(device="cuda").manual_seed(7)
        mk = lambda *s: torch.randn(s, device="cuda", generator=g).to(BF)
        self.mods, self.B, self.T, self.page = (G, P, R, K), B, B * n, page
        T, most, P_ = self.T, 12, 120
        self.kv = mk(2, 2, P_, KH, page, D)
        self.layers = [[mk(T, H, D), mk(T, KH, D), mk(T, KH, D), G.KVCache(x[0], x[1]),
                        torch.zeros((T, H, D), dtype=BF, device="cuda")] for x in self.kv]
        self.caches = K.Caches([x[3] for x in self.layers])
        self.past, self.new = i32([0] * B), i32([0] * B)
        self.parent, self.given = i32([-1] * T), i32([1] * B)
        self.drafted = torch.zeros(T, dtype=I64, device="cuda")
        self.target = torch.zeros(T, dtype=I64, device="cuda")
        # prompts of 3 and 2 pages, held by two requests each and their adapter
        self.group, self.prefix = i32([0, 0, 1, 1, -1, -1]), i32([48, 32])
        perm = np.random.default_rng(1).permutation(P_)
        table = np.full((B, most), -1)
        lead = [perm[:3], perm[3:5]]
        at, shares = 5, np.zeros(P_, int)
        for b, grp in enumerate([0, 0, 1, 1, -1, -1]):
            k = 0
            if grp >= 0:
                k = len(lead[grp])
                table[b, :k] = lead[grp]
                shares[lead[grp]] = 2
            table[b, k:6] = perm[at:at + 6 - k]
            at += 6 - k
        self.table = i32(table)
        self.pool = K.PagePool(i32(shares), i32(np.r_[[-1] * 30, perm[at:]]))
        self.h0, self.h1, self.h2 = i32([30]), i32([0]), i32([0])
        self.step = G.Step(B, T, page, most, table=self.table)
        self.tree = R.Tree(self.step)
        self.plan = G.AttnPlan(self.step, H, KH, D, max_q=n, shared=True)
        self.segs = P.Segments(B, 2)
        self.acc = R.Accepted(self.step, dtype=I64)
        self.src = i32(range(B))
        self.out = K.Remap(B, B, page, most)
        self.turns = G.rope_turns(D)
        self.state = [self.kv, self.table, self.pool.shares, self.pool.free_pages, self.out.table,
                      self.out.kv_len, self.out.copies, self.out.meta, self.h1, self.h2,
                      self.acc.path, self.acc.count, self.acc.token, self.acc.kv_len,
                      self.tree.pos, self.tree.span, self.tree.info]
        self.state += [t for x in self.layers for t in (x[0], x[4])]
        self.keep = [t.clone() for t in self.state]

    def reset(self):
        for t, k in zip(self.state, self.keep):
            t.copy_(k)

    def fill(self, rng, kinds):
        """Other lengths, trees and tokens in the same buffers."""
        lens = rng.integers(49, 96, self.B)
        new = rng.integers(0, 21, self.B)
        par = np.full(self.T, -1)
        at = 0
        for b, n in enumerate(new):
            par[at:at + n] = shape_of(kinds[b % len(kinds)], int(n), rng)
            at += n
        self.past.copy_(i32(lens)), self.new.copy_(i32(new)), self.parent.copy_(i32(par))
        tok = lambda: torch.from_numpy(rng.integers(0, 3, self.T)).cuda()
        self.drafted.copy_(tok()), self.target.copy_(tok())
        self.given.copy_(i32(rng.integers(0, 3, self.B)))

    def call(self, stream=None):
        G, P, R, K = self.mods
        kw = dict(stream=stream)
        G.kv_plan(self.past, self.new, self.pool.free_pages, self.h0, self.h1, self.step, **kw)
        R.tree_plan(self.parent, self.step, self.tree, **kw)
        P.segment(self.group, self.segs, **kw)
        G.attn_plan(self.step, self.plan, self.segs, self.prefix, **kw)
        R.run_layers(self.step, self.plan, self.tree, self.layers, self.turns, 0.125, **kw)
        R.tree_accept(self.parent, self.drafted, self.target, self.step, self.acc, self.given, **kw)
        K.kv_compact(self.caches, self.step, self.acc.path, self.acc.count, **kw)
        K.kv_remap(self.table, self.step.kv_len, self.src, self.acc.kv_len, self.pool, self.h1,
                   self.h2, self.out, **kw)
        K.kv_copy(self.caches, self.out, **kw)


def test_captured_and_replayed(G, P, R, K):
    s = Step(G, P, R, K)
    rng = np.random.default_rng(5)
    s.fill(rng, ["levels"])
    s.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    for kinds in (["levels", "any"], ["chain"], ["star", "bad", "comb"], ["roots", "levels"]):
        s.fill(rng, kinds)
        s.reset()
        s.call()
        want = [t.clone() for t in s.state]
        for _ in range(2):
            s.reset()
            graph.replay()
            torch.cuda.synchronize()
            for t, w in zip(s.state, want):
                assert torch.equal(t, w)


def test_on_a_stream_of_the_callers(G, P, R, K):
    s = Step(G, P, R, K)
    rng = np.random.default_rng(6)
    s.fill(rng, ["levels", "any"])
    s.reset()
    s.call()
    torch.cuda.synchronize()
    want = [t.clone() for t in s.state]
    other = torch.cuda.Stream()
    s.reset()
    torch.cuda.synchronize()
    s.call(stream=other)
    other.synchronize()
    for t, w in zip(s.state, want):
        assert torch.equal(t, w)


def refused(call, args):
    """Runs with all on the GPU, then with each argument on the host in turn."""
    call(**args)
    torch.cuda.synchronize()
    for name, t in args.items():
        with pytest.raises(ValueError, match="device"):
            call(**dict(args, **{name: t.cpu()}))


def test_each_argument_is_on_the_gpu(G, P, R, K):
    z = lambda *s, dt=BF: torch.zeros(s, dtype=dt, device="cuda")
    i = lambda *n, dt=I32: torch.zeros(n, dtype=dt, device="cuda")
    step = G.Step(2, 5, 16, 4)
    tree, acc = R.Tree(step), R.Accepted(step)
    refused(lambda **a: R.tree_plan(a["parent"], step, tree), dict(parent=i(5)))
    refused(lambda **a: R.tree_accept(a["parent"], a["drafted"], a["target"], step, acc, a["given"]),
            dict(parent=i(5), drafted=i(5), target=i(5), given=i(2)))
    cache = G.KVCache(z(3, 2, 16, 64), z(3, 2, 16, 64))
    plan = G.AttnPlan(step, 4, 2, 64, max_q=3)
    G.attn_plan(step, plan)
    refused(lambda **a: R.attn_tree(a["q"], cache, step, plan, tree, 0.1, a["out"]),
            dict(q=z(5, 4, 64), out=z(5, 4, 64)))
    caches = K.Caches([cache])
    refused(lambda **a: K.kv_compact(caches, step, a["path"], a["count"]),
            dict(path=i(5), count=i(2)))
    pool, out = K.PagePool(i(3), i(3)), K.Remap(2, 3, 16, 4)
    refused(lambda **a: K.kv_remap(a["table"], a["kv_len"], a["src"], a["keep"], pool, a["head"],
                                   a["next"], out),
            dict(table=i(2, 4), kv_len=i(2), src=i(3), keep=i(3), head=i(1), next=i(1)))
    K.kv_copy(caches, out)
    # and what the calls are given beside tensors
    host = G.Step(2, 5, 16, 4, device="cpu")
    cold = G.KVCache(cache.k.cpu(), cache.v.cpu())
    q = z(5, 4, 64)
    for call in (lambda: R.tree_plan(i(5), host, tree),
                 lambda: R.tree_plan(i(5), step, R.Tree(step, device="cpu")),
                 lambda: R.tree_accept(i(5), i(5), i(5), host, acc),
                 lambda: R.tree_accept(i(5), i(5), i(5), step, R.Accepted(step, device="cpu")),
                 lambda: R.attn_tree(q, cache, step, plan, R.Tree(step, device="cpu"), 0.1, q),
                 lambda: R.attn_tree(q, cold, step, plan, tree, 0.1, q),
                 lambda: K.Caches([cache, cold]),
                 lambda: K.kv_compact(caches, host, i(5), i(2)),
                 lambda: K.kv_copy(caches, K.Remap(2, 3, 16, 4, device="cpu")),
                 lambda: K.kv_remap(i(2, 4), i(2), i(3), None, K.PagePool(i(3).cpu(), i(3).cpu()),
                                    i(1), i(1), out),
                 lambda: K.PagePool(i(3), i(3).cpu())):
        with pytest.raises(ValueError, match="device"):
            call()
