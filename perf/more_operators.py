"""The work of a serving step that verifies trees of drafted tokens, and of the
cache's upkeep around it, as cases that can be timed and compared.

A case is one of five kinds of pass:

  tree     the layout of a step's trees, built on the GPU from each node's parent:
           rotary positions by depth, and the interval of preorder numbers that a
           node's descendants have.  Once a step.
  attn     one layer's attention over the paged cache, in which a drafted token
           sees the request's cached keys and its own ancestors.  The step's plan
           is in hand, as it serves every layer.
  accept   which path of each tree the model's choices follow, and the token
           behind it.  Once a step.
  compact  the keys of the accepted nodes moved together, in the caches of all
           layers.  Once a step.
  fork     every request continued by several (shared pages counted, the partly
           filled one copied in all layers), then all but one of them dropped and
           their pages given back: sampling of a few continuations for one token.

Where ``own`` is false the operators are computed in their plain form, from
elementary torch operations in 32 bits and whole numbers; where it is true,
through the public entry points of ``paper_2608_05483_amd.tree`` and ``.pages``.

Batches, head counts and lengths are those of the framework's decode and prompt
workloads: 64 requests of 512 to 4096 keys, prompts of up to 512 tokens, a few long
contexts on 8 key heads, heads of 128 and 64, and trees of 1 to a few hundred nodes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "int32": torch.int32,
          "int64": torch.int64}
VOCAB = 32000


def listed():
    return [
        # trees of 20..60 nodes for the benchmark's batch of 64 requests
        dict(name="tree_64", kind="tree", batch=64, past_lo=511, past_hi=4095, nodes_lo=20,
             nodes_hi=60, branch=3, prompts=0, page=16),
        # a large mixed batch: small and larger trees, one request in eight a chunk of
        # a prompt (a chain of up to 500 tokens)
        dict(name="tree_mixed_400", kind="tree", batch=400, past_lo=0, past_hi=8000, nodes_lo=1,
             nodes_hi=100, branch=4, prompts=500, page=64),
        # one user with a long context and a tree of 48, grouped-query
        dict(name="attn_tree_one", kind="attn", batch=1, past_lo=30010, past_hi=30010,
             nodes_lo=48, nodes_hi=48, branch=4, prompts=0, groups=0, prefix=0, heads=64,
             kv_heads=8, d=128, page=16, dtype="bf16"),
        # the benchmark's decode batch, each request with a tree of 8..24
        dict(name="attn_tree_64", kind="attn", batch=64, past_lo=511, past_hi=4095, nodes_lo=8,
             nodes_hi=24, branch=3, prompts=0, groups=0, prefix=0, heads=32, kv_heads=32, d=128,
             page=16, dtype="bf16"),
        # small trees of a large batch in which each adapter's requests start with its prompt
        dict(name="attn_tree_shared_128", kind="attn", batch=128, past_lo=1, past_hi=511,
             nodes_lo=4, nodes_hi=13, branch=2, prompts=0, groups=6, prefix=4000, heads=64,
             kv_heads=8, d=128, page=32, dtype="fp16"),
        # few requests with the largest trees beside chunks of prompts, heads of 64: bound
        # by the products
        dict(name="attn_tree_wide_24", kind="attn", batch=24, past_lo=500, past_hi=6000,
             nodes_lo=100, nodes_hi=250, branch=6, prompts=700, groups=0, prefix=0, heads=32,
             kv_heads=8, d=64, page=64, dtype="bf16"),
        # one request's tree of 30: the smallest call
        dict(name="accept_one", kind="accept", batch=1, past_lo=700, past_hi=700, nodes_lo=30,
             nodes_hi=30, branch=3, prompts=0, page=16, dtype="int64"),
        # a large batch of trees and prompts
        dict(name="accept_1000", kind="accept", batch=1000, past_lo=0, past_hi=4000, nodes_lo=1,
             nodes_hi=60, branch=3, prompts=300, page=16, dtype="int32"),
        # one request's accepted path in 32 layers
        dict(name="compact_one", kind="compact", batch=1, past_lo=700, past_hi=700, nodes_lo=30,
             nodes_hi=30, most=6, layers=32, kv_heads=8, d=128, page=16, dtype="bf16"),
        # the paths of 64 requests in 16 layers
        dict(name="compact_64", kind="compact", batch=64, past_lo=33, past_hi=200, nodes_lo=20,
             nodes_hi=60, most=9, layers=16, kv_heads=8, d=128, page=16, dtype="fp16"),
        # one prompt continued by 8 samples
        dict(name="fork_one", kind="fork", batch=1, past_lo=4011, past_hi=4011, samples=8,
             groups=0, prefix=0, layers=32, kv_heads=8, d=128, page=16, dtype="bf16"),
        # 64 requests behind their adapters' prompts, 4 samples each, pages of 64 keys
        dict(name="fork_64", kind="fork", batch=64, past_lo=60, past_hi=900, samples=4, groups=5,
             prefix=1000, layers=6, kv_heads=8, d=128, page=64, dtype="bf16"),
    ]


# ---- more cases of the same ranges --------------------------------------------------

HEADS = ((32, 32), (40, 40), (64, 8), (32, 8), (16, 16), (16, 1), (40, 8), (12, 4), (8, 8))


def _loguni(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a, b = sorted((_loguni(rng, max(lo, 1), hi), _loguni(rng, max(lo, 1), hi)))
    return (lo if rng.random() < 0.2 else a, b)


def _drawn_nodes(rng, batch, most):
    lo, hi = _range(rng, 1, max(2, most))
    return dict(nodes_lo=lo, nodes_hi=hi, branch=rng.randint(1, 8))


def draw(rng):
    kind = rng.choice(["tree", "attn", "attn", "attn", "attn", "accept", "compact", "fork"])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind in ("tree", "accept"):
        batch = _loguni(rng, 1, 1000)
        # (the plain form's matrices of ancestors: 400 of 512 x 512 at most)
        most = int(min(300, (1e8 / batch) ** 0.5))
        past = _range(rng, 0, 30000)
        prompts = _loguni(rng, 2, max(2, most)) if rng.random() < 0.4 else 0
        return dict(kind=kind, batch=batch, past_lo=past[0], past_hi=past[1], page=page,
                    prompts=prompts, dtype=rng.choice(["int32", "int64"]),
                    **_drawn_nodes(rng, batch, most))
    if kind == "compact":
        batch, layers = _loguni(rng, 1, 200), rng.randint(1, 32)
        kv_heads, d = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.choice([128, 128, 64, 80])
        past = _range(rng, 0, 400)
        nodes = _drawn_nodes(rng, batch, 120)
        c = dict(kind=kind, batch=batch, past_lo=past[0], past_hi=past[1], layers=layers,
                 kv_heads=kv_heads, d=d, page=page, most=rng.randint(2, 12),
                 nodes_lo=nodes["nodes_lo"], nodes_hi=nodes["nodes_hi"],
                 dtype=rng.choice(["bf16", "fp16"]))
        # no dearer than the listed ones: pools of 0.7 GB in all
        while c["batch"] * (c["past_hi"] + c["nodes_hi"] + page) * kv_heads * d * 4.0 * \
                c["layers"] > 7e8:
            if c["layers"] > 1:
                c["layers"] = c["layers"] * 3 // 4
            else:
                c["batch"] = max(1, c["batch"] * 3 // 4)
        return c
    if kind == "fork":
        batch, samples = _loguni(rng, 1, 100), rng.randint(2, 9)
        groups = min(batch, rng.choice([0, 1, rng.randint(2, 9)]))
        past = _range(rng, 1, 4000)
        c = dict(kind=kind, batch=batch, past_lo=past[0], past_hi=past[1], samples=samples,
                 groups=groups, prefix=_loguni(rng, 20, 2000) if groups else 0,
                 layers=rng.randint(1, 32), kv_heads=rng.choice([1, 2, 4, 8, 8, 32]),
                 d=rng.choice([128, 128, 64, 80]), page=page, dtype=rng.choice(["bf16", "fp16"]))
        # pools of 1.2 GB in all
        while (c["batch"] * (c["past_hi"] + page * samples) + groups * c["prefix"]) * 4.0 * \
                c["kv_heads"] * c["d"] * c["layers"] > 1.2e9:
            if c["layers"] > 4:
                c["layers"] = c["layers"] * 3 // 4
            elif c["past_hi"] > 200:
                c["past_lo"], c["past_hi"] = c["past_lo"] * 3 // 4 + 1, c["past_hi"] * 3 // 4
                c["past_lo"] = min(c["past_lo"], c["past_hi"])
            else:
                c["batch"] = max(1, c["batch"] * 3 // 4)
                c["groups"] = groups = min(groups, c["batch"])
                c["layers"] = max(1, c["layers"] - 1)
        return c
    heads, kv_heads = rng.choice(HEADS)
    d = rng.choice([128, 128, 128, 64])
    form = rng.choice(["few", "few", "middle", "wide"])
    if form == "few":
        batch, most = _loguni(rng, 1, 256), rng.randint(2, 16)
    elif form == "middle":
        batch, most = _loguni(rng, 1, 100), rng.randint(8, 64)
    else:
        batch, most = _loguni(rng, 1, 24), rng.randint(32, 300)
    groups = rng.choice([0, 0, 1, rng.randint(2, 9)]) if batch > 1 else 0
    groups = min(groups, batch)
    prefix = _loguni(rng, 20, 4096) if groups else 0
    past = _range(rng, 0, 30000)
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, d=d, page=page, batch=batch,
             dtype=rng.choice(["bf16", "bf16", "fp16"]), groups=groups, prefix=prefix,
             past_lo=past[0], past_hi=past[1],
             prompts=rng.randint(16, 700) if form == "wide" and rng.random() < 0.5 else 0,
             **_drawn_nodes(rng, batch, most))
    # no dearer than the listed ones: caches of 2.2 GB, 0.6 TFLOP, 2 GB of scores
    def too_dear():
        new = max(c["nodes_hi"], c["prompts"])
        keys = c["past_hi"] + new
        rows = c["batch"] * ((c["nodes_lo"] + c["nodes_hi"]) / 2 + c["prompts"] / 8) * heads
        return (c["batch"] * keys * kv_heads * d * 4 > 2.2e9
                or rows * (prefix + keys) * d * 4 > 6e11
                or (prefix + keys) * heads * new * 4 > 2e9)
    while too_dear():
        if c["past_hi"] > 4:
            c["past_lo"], c["past_hi"] = c["past_lo"] * 3 // 4, c["past_hi"] * 3 // 4
        else:
            c["batch"] = max(1, c["batch"] * 3 // 4)
            c["groups"] = min(c["groups"], c["batch"])
    return c


# ---- inputs -------------------------------------------------------------------------


class State:
    pass


def _rng(case, seed):
    return np.random.default_rng([seed, case["batch"], 29])


def _spread(lo, hi, n, rng):
    """n whole numbers over [lo, hi], one of each n-th part."""
    u = (rng.permutation(n) + rng.random(n)) / n
    return np.minimum(hi, np.floor(lo + u * (hi + 1 - lo))).astype(np.int64)


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=gen)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=dtype)


def _tree(n, branch, rng):
    """Parents of a drafted tree of n nodes in the order of their levels: each node
    has up to ``branch`` children, the last one of a level at least one."""
    parent, at, left = [-1], 0, 1 + int(rng.integers(branch))
    while len(parent) < n:
        if left == 0:
            at += 1
            left = int(rng.integers(branch + 1))
            if at == len(parent) - 1:
                left = max(left, 1)
            continue
        parent.append(at)
        left -= 1
    return np.array(parent[:n], np.int64)


def _lengths(case):
    """Which requests there are is part of the case, so that every seed asks for the
    same work: keys held, new tokens, which are chunks of prompts, groups."""
    rng = _rng(case, 0)
    B = case["batch"]
    past = _spread(case["past_lo"], case["past_hi"], B, rng) + case.get("prefix", 0)
    new = _spread(case["nodes_lo"], case["nodes_hi"], B, rng) if "nodes_lo" in case else \
        np.zeros(B, np.int64)
    chunk = np.zeros(B, bool)
    if case.get("prompts"):
        chunk[rng.permutation(B)[:(B + 7) // 8]] = True
        new = np.where(chunk, _spread(1, case["prompts"], B, rng), new)
    group = np.full(B, -1, np.int64)
    G = case.get("groups", 0)
    if G:
        # requests fall to the groups unevenly; one in sixteen belongs to none and
        # holds a prefix of its own
        w = 1.0 / np.arange(1, G + 1)
        group = rng.choice(G, size=B, p=w / w.sum())
        group[rng.random(B) < 1 / 16] = -1
    return past, new, chunk, group


def _batch(case, seed, spare=0):
    """The step's requests; their order, trees and pages are the seed's."""
    s = State()
    s.case, s.B, s.page = case, case["batch"], case["page"]
    s.G, s.prefix = case.get("groups", 0), case.get("prefix", 0)
    past, new, chunk, group = _lengths(case)
    rng = _rng(case, seed + 1)
    order = rng.permutation(s.B)
    s.past, s.new, s.chunk, s.group = past[order], new[order], chunk[order], group[order]
    s.kv, s.T = s.past + s.new, int(s.new.sum())
    s.starts = np.concatenate([[0], np.cumsum(s.new)])
    S = s.page
    s.max_pages = int(-(-s.kv.max() // S)) + 1
    pages = -(-s.kv // S)
    whole = s.prefix // S
    s.n_pages = int(s.G * whole + pages.sum()) + 8 + spare
    ids = rng.permutation(s.n_pages)
    at = s.G * whole
    table = np.zeros((s.B, s.max_pages), np.int64)
    for b in range(s.B):
        lead = 0
        if s.group[b] >= 0:
            table[b, :whole] = ids[s.group[b] * whole:(s.group[b] + 1) * whole]
            lead = whole
        n = int(pages[b]) - lead
        table[b, lead:lead + n] = ids[at:at + n]
        at += n
    s.table, s.free, s.rng = table, ids[at:], rng
    return s


def _trees(s):
    """Each request's parents, one after another: a tree, or a chunk's chain."""
    c = s.case
    s.trees = [np.arange(n) - 1 if c else _tree(int(n), s.case["branch"], s.rng)
               for n, c in zip(s.new, s.chunk)]
    s.parent = np.concatenate(s.trees)
    s.d_parent = _dev(s.parent)


def _place(s):
    """The batch's arrays on the GPU, as the step's layout leaves them."""
    s.d_table, s.d_start, s.d_past = _dev(s.table), _dev(s.starts), _dev(s.past)
    s.d_req = _dev(np.repeat(np.arange(s.B), s.new))
    s.n_max = int(s.new.max())


def _step(s):
    """The step that a user's program has planned."""
    from paper_2608_05483_amd import paged
    s.step = paged.Step(s.B, s.T, s.page, s.max_pages, device=DEV, table=s.d_table.clone())
    z = lambda: torch.zeros(1, dtype=torch.int32, device=DEV)
    # the pages are in the table; a list of the same ones hands them out again
    held, kept = -(-s.past // s.page), -(-s.kv // s.page)
    free = np.concatenate([s.table[b, held[b]:kept[b]] for b in range(s.B)] + [s.free])
    paged.kv_plan(s.d_past, _dev(s.new), _dev(free), z(), z(), s.step)


def _caches(s, gen, layers):
    """All layers' pools in one tensor: [layers, k or v, pages, key heads, page, dim]."""
    case = s.case
    s.kv_pool = _normal((layers, 2, s.n_pages, case["kv_heads"], s.page, case["d"]),
                        DTYPES[case["dtype"]], gen)


def _inputs(case, seed):
    """Everything but the framework's handles."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    if kind == "fork":
        return _fork_inputs(case, seed, gen)
    s = _batch(case, seed)
    _place(s)
    if kind == "compact":
        return _compact_inputs(s, gen)
    _trees(s)
    if kind == "accept":
        _accept_inputs(s)
    if kind == "attn":
        H, D = case["heads"], case["d"]
        s.q = _normal((s.T, H, D), DTYPES[case["dtype"]], gen)
        s.out = torch.zeros_like(s.q)
        _caches(s, gen, 1)
        s.scale = D ** -0.5
        if s.G:
            s.d_group = _dev(s.group)
            s.d_prefix = torch.full((s.G,), s.prefix, dtype=torch.int32, device=DEV)
    return s


def _accept_inputs(s):
    """Drafted tokens (siblings differ) and the model's choice behind each node: a
    child's token for seven of ten nodes that have children.  The tokens of a prompt's
    chunk are given, of a tree the first."""
    rng = s.rng
    drafted = rng.integers(0, VOCAB, s.T)
    target = rng.integers(0, VOCAB, s.T)
    for b in range(s.B):
        lo, par = int(s.starts[b]), s.trees[b]
        n = len(par)
        # a child's token: its parent's base plus its own number
        drafted[lo:lo + n] = (drafted[lo] + 7 * par + np.arange(n)) % VOCAB
        if n > 1:
            kids = 1 + rng.permutation(n - 1)
            pick = kids[rng.random(n - 1) < 0.9]
            target[lo + par[pick]] = drafted[lo + pick]
            stop = rng.random(n) < 0.22
            target[lo:lo + n][stop] = (drafted[lo] + 7 * n + 11 * n) % VOCAB
    dt = DTYPES[s.case["dtype"]]
    s.d_drafted, s.d_target = _dev(drafted, dt), _dev(target, dt)
    s.drafted, s.target = drafted, target
    # levels of the deepest drafted tree
    s.levels = 0
    for c, par in zip(s.chunk, s.trees):
        depth = np.zeros(len(par), np.int64)
        for i in range(1, 0 if c else len(par)):
            depth[i] = depth[par[i]] + 1
        s.levels = max(s.levels, int(depth.max()))
    s.given = np.where(s.chunk, s.new, 1)
    s.d_given = _dev(s.given)


def _compact_inputs(s, gen):
    """Accepted paths: the first node, then by chance the next few in their places
    already, then nodes further on.  (No moved key lands where another moved from, so
    that the same pass can be made again.)"""
    case, rng = s.case, s.rng
    s.path = np.full(s.T, -1, np.int64)
    s.count = np.zeros(s.B, np.int64)
    for b in range(s.B):
        n, lo = int(s.new[b]), int(s.starts[b])
        a = min(1 + int(rng.integers(case["most"])), (n + 1) // 2)
        stay = 1 + int(rng.integers(a))
        stay = max(stay, 2 * a - n)
        far = np.sort(rng.permutation(n - a)[:a - stay]) + a
        s.path[lo:lo + a] = np.concatenate([np.arange(stay), far])
        s.count[b] = a
    s.d_path, s.d_count = _dev(s.path), _dev(s.count)
    _caches(s, gen, case["layers"])
    return s


def _fork_inputs(case, seed, gen):
    k, B = case["samples"], case["batch"]
    s = _batch(case, seed, spare=B * k)
    s.k = k
    _place(s)
    _caches(s, gen, case["layers"])
    # holders of a page beyond the first: the adapters' prompts are held by the
    # adapter and by its requests
    held = np.zeros(s.n_pages, np.int64)
    for b in range(B):
        held[s.table[b, :-(-s.kv[b] // s.page)]] += 1
    if s.G:
        whole = s.prefix // s.page
        first = {int(g): b for b, g in reversed(list(enumerate(s.group))) if g >= 0}
        for b in first.values():
            held[s.table[b, :whole]] += 1
    s.shares = np.maximum(held - 1, 0)
    s.d_shares = _dev(s.shares)
    # entries before the list's head have been handed out
    s.lead = 5
    s.free_list = np.concatenate([np.zeros(s.lead, np.int64), s.free])
    s.d_free = _dev(s.free_list)
    s.d_len = _dev(s.kv)
    # request b is continued by k b .. k b + k - 1, and those by their last one
    s.src, s.back = np.repeat(np.arange(B), k), np.arange(B) * k + k - 1
    s.d_src, s.d_back = _dev(s.src), _dev(s.back)
    z = lambda v: torch.full((1,), v, dtype=torch.int32, device=DEV)
    s.d_head, s.d_next, s.d_next2 = z(s.lead), z(0), z(0)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if not own:
        if kind == "attn":
            s.seen = _plain_seen(s)
        if kind == "fork":
            s.out1, s.out2 = _plain_remap_buffers(s, s.B * s.k), _plain_remap_buffers(s, s.B)
        if kind in ("accept", "compact"):
            s.d_slot = _plain_slots(s)
        return s
    from paper_2608_05483_amd import paged, pages, plora, tree
    if kind == "fork":
        s.pool = pages.PagePool(s.d_shares, s.d_free)
        s.caches = pages.Caches([paged.KVCache(x[0], x[1]) for x in s.kv_pool])
        s.out1 = pages.Remap(s.B, s.B * s.k, s.page, s.max_pages, device=DEV)
        s.out2 = pages.Remap(s.B * s.k, s.B, s.page, s.max_pages, device=DEV)
        return s
    _step(s)
    if kind == "compact":
        s.caches = pages.Caches([paged.KVCache(x[0], x[1]) for x in s.kv_pool])
    if kind in ("tree", "attn"):
        s.tree = tree.Tree(s.step, device=DEV)
    if kind == "accept":
        s.accepted = tree.Accepted(s.step, dtype=DTYPES[case["dtype"]], device=DEV)
    if kind == "attn":
        s.cache = paged.KVCache(s.kv_pool[0, 0], s.kv_pool[0, 1])
        s.plan = paged.AttnPlan(s.step, case["heads"], case["kv_heads"], case["d"],
                                max_q=s.n_max, shared=bool(s.G), device=DEV)
        tree.tree_plan(s.d_parent, s.step, s.tree)
        if s.G:
            s.segs = plora.Segments(s.B, s.G, device=DEV)
            plora.segment(s.d_group, s.segs)
            paged.attn_plan(s.step, s.plan, s.segs, s.d_prefix)
        else:
            paged.attn_plan(s.step, s.plan)
    return s


# ---- plain forms --------------------------------------------------------------------


def _plain_rows(s):
    """A row of the batch's tokens for every request, and which of them there are."""
    i = torch.arange(s.n_max, device=DEV)
    at = s.d_start[:-1, None].long() + i[None, :]
    there = at < s.d_start[1:, None]
    return at.clamp(max=s.T - 1), there, i


def _plain_ancestors(par, i):
    """[requests, nodes, nodes] 1.0 where the second is an ancestor of the first or
    itself: paths of twice the length by each product."""
    n = i.numel()
    m = (par[:, :, None] == i[None, None, :]).float() + torch.eye(n, device=DEV)
    length = 1
    while length < n:
        m = torch.bmm(m, m.contiguous()).clamp(max=1.0)
        length *= 2
    return m


def _plain_tree(s):
    at, there, i = _plain_rows(s)
    par = torch.where(there, s.d_parent[at].long(), torch.full_like(at, -9))
    m = _plain_ancestors(par, i)
    depth, size = m.sum(2) - 1.0, m.sum(1)
    sib = (par[:, :, None] == par[:, None, :]) & (i[None, None, :] < i[None, :, None])
    before = (sib & there[:, None, :]).float()
    before = torch.bmm(before, size[:, :, None].contiguous())
    first = (depth + torch.bmm(m, before)[:, :, 0]).long()
    last = first + size.long() - 1
    chain = ((par == i[None, :] - 1) | ~there).all(1)
    pos = s.d_past[:, None].long() + depth.long()
    span = torch.stack([first, last], -1)
    info = torch.stack([(~chain).int(), torch.zeros_like(chain, dtype=torch.int32)], -1)
    return {"pos": pos[there].int(), "span": span[there].int(), "info": info}


def _plain_seen(s):
    """Each request's matrix of which new keys its new tokens see."""
    out = []
    for b in range(s.B):
        i = torch.arange(int(s.new[b]), device=DEV)
        par = s.d_parent[int(s.starts[b]):int(s.starts[b + 1])].long()
        out.append(_plain_ancestors(par[None], i)[0] > 0)
    return out


def _plain_attention(s):
    """Request by request in 32 bits."""
    q, kp, vp = s.q, s.kv_pool[0, 0], s.kv_pool[0, 1]
    H, D = q.shape[1:]
    KH = kp.shape[1]
    r = H // KH
    out = torch.zeros_like(q)
    for b in range(s.B):
        lo, hi, n = int(s.starts[b]), int(s.starts[b + 1]), int(s.kv[b])
        m = hi - lo
        pages = s.d_table[b, :-(-n // s.page)].long()
        K = kp[pages].transpose(0, 1).reshape(KH, -1, D)[:, :n].float()
        V = vp[pages].transpose(0, 1).reshape(KH, -1, D)[:, :n].float()
        qb = q[lo:hi].float().view(m, KH, r, D).permute(1, 2, 0, 3)
        w = torch.matmul(qb.reshape(KH, r * m, D), K.transpose(1, 2).contiguous()) * s.scale
        w = w.view(KH, r, m, n)
        w[..., n - m:].masked_fill_(~s.seen[b], -math.inf)
        w -= w.amax(-1, keepdim=True)
        w = torch.exp(w)
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w.view(KH, r * m, n), V.contiguous()).view(KH, r, m, D) / total
        out[lo:hi] = o.permute(2, 0, 1, 3).reshape(m, H, D).to(q.dtype)
    return {"out": out}


def _plain_accept(s):
    """All requests a node at a time."""
    at, there, i = _plain_rows(s)
    par = torch.where(there, s.d_parent[at].long(), torch.full_like(at, -9))
    drafted = s.d_drafted[at]
    start = s.d_start[:-1].long()
    some = s.d_start[1:] > s.d_start[:-1]
    given = torch.minimum(s.d_given, s.d_start[1:] - s.d_start[:-1]).long()
    path = torch.where(i[None, :] < given[:, None], i[None, :], torch.full_like(at, -1))
    cur = (given - 1).clamp(min=0)
    count, going = given.clone(), some
    for _ in range(s.levels):
        want = s.d_target[(start + cur).clamp(max=s.T - 1)]
        fits = (par == cur[:, None]) & (drafted == want[:, None]) & there
        going = going & fits.any(1)
        child = torch.where(fits, i[None, :], torch.full_like(at, s.n_max)).amin(1)
        cur = torch.where(going, child, cur)
        put = going[:, None] & (i[None, :] == count[:, None])
        path = torch.where(put, cur[:, None], path)
        count = count + going.long()
    token = torch.where(some, s.d_target[(start + cur).clamp(max=s.T - 1)].long(),
                        torch.full_like(cur, -1))
    return {"path": path[there].int(), "count": count.int(), "token": token.to(s.d_target.dtype),
            "kv_len": (s.d_past.long() + count).int()}


def _plain_slots(s):
    req = s.d_req.long()
    pos = s.d_past[req].long() + torch.arange(s.T, device=DEV) - s.d_start[req].long()
    return s.d_table[req, pos // s.page].long() * s.page + pos % s.page


def _plain_compact(s):
    req, S = s.d_req.long(), s.page
    rank = torch.arange(s.T, device=DEV) - s.d_start[req].long()
    moves = (rank < s.d_count[req]) & (s.d_path.long() != rank)
    src = s.d_slot[(s.d_start[req].long() + s.d_path.long())[moves]]
    dst = s.d_slot[moves]
    for x in s.kv_pool:
        for pool in x:
            pool[dst // S, :, dst % S] = pool[src // S, :, src % S]
    return {"kv": s.kv_pool}


def _plain_remap_buffers(s, n):
    o = State()
    i32 = dict(dtype=torch.int32, device=DEV)
    o.table = torch.zeros((n, s.max_pages), **i32)
    o.kv_len, o.meta = torch.zeros(n, **i32), torch.zeros(8, **i32)
    o.copies = torch.full((n, 3), -1, **i32)
    return o


def _plain_remap(s, table, kv_len, src, head, nxt, o):
    """The new batch, all pages at once.  Keeps whole requests."""
    S, n, P = s.page, src.numel(), s.n_pages
    j = torch.arange(s.max_pages, device=DEV)[None, :]
    src = src.long()
    keep = kv_len[src].long()
    new = table[src].long()
    old_held = j < ((kv_len.long() + S - 1) // S)[:, None]
    held = j < ((keep + S - 1) // S)[:, None]
    old = table.long()[old_held]
    shares = s.d_shares.long()
    shares.index_add_(0, new[held], torch.ones_like(new[held]))
    shares.index_add_(0, old, -torch.ones_like(old))
    # pages without a holder, each once, in the old requests' order
    flat = torch.arange(old.numel(), device=DEV)
    first = torch.full((P,), old.numel(), device=DEV, dtype=torch.int64)
    first.scatter_reduce_(0, old, flat, "amin")
    gone = (shares[old] < 0) & (first[old] == flat)
    freed = old[gone]
    shares.clamp_(min=0)
    top = head.long() - freed.numel()
    s.d_free[top + torch.arange(freed.numel(), device=DEV)] = freed.int()
    # partly filled pages of several holders: in the requests' order, each but the
    # last holder takes a page of its own
    part = keep % S != 0
    at = (keep // S).clamp(max=s.max_pages - 1)
    page = new.gather(1, at[:, None])[:, 0]
    i = torch.arange(n, device=DEV)
    same = (page[:, None] == page[None, :]) & part[None, :] & (i[None, :] < i[:, None])
    own_copy = part & (shares[page] + 1 - same.sum(1) > 1)
    rank = torch.cumsum(own_copy.long(), 0) - 1
    fresh = s.d_free[(top + rank).clamp(0, s.d_free.numel() - 1)].long()
    shares.index_add_(0, page[own_copy], -torch.ones_like(page[own_copy]))
    copies = torch.stack([page, fresh, keep % S], 1)[own_copy]
    new.scatter_(1, at[:, None], torch.where(own_copy, fresh, page)[:, None])
    o.table.copy_(torch.where(held, new, o.table.long()))
    o.kv_len.copy_(keep)
    o.copies.fill_(-1)
    o.copies[:copies.shape[0]] = copies.int()
    o.meta.zero_()
    o.meta[0], o.meta[1] = freed.numel(), copies.shape[0]
    s.d_shares.copy_(shares)
    nxt.copy_(top + copies.shape[0])
    return copies.long()


def _plain_fork(s):
    copies = _plain_remap(s, s.d_table, s.d_len, s.d_src, s.d_head, s.d_next, s.out1)
    k = torch.arange(s.page, device=DEV)[None, :]
    some = k < copies[:, 2:]
    e, key = some.nonzero(as_tuple=True)
    for x in s.kv_pool:
        for pool in x:
            pool[copies[e, 1], :, key] = pool[copies[e, 0], :, key]
    _plain_remap(s, s.out1.table, s.out1.kv_len, s.d_back, s.d_next, s.d_next2, s.out2)
    return _fork_outputs(s)


def _fork_outputs(s):
    f = lambda o, nxt: {"table": o.table, "kv_len": o.kv_len, "copies": o.copies,
                        "meta": o.meta, "next": nxt}
    return {"forked": f(s.out1, s.d_next), "kept": f(s.out2, s.d_next2), "shares": s.d_shares,
            "free": s.d_free, "kv": s.kv_pool}


# ---- one pass -----------------------------------------------------------------------


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"tree": _plain_tree, "attn": _plain_attention, "accept": _plain_accept,
                "compact": _plain_compact, "fork": _plain_fork}[kind](s)
    from paper_2608_05483_amd import pages, tree
    if kind == "tree":
        tree.tree_plan(s.d_parent, s.step, s.tree)
        return {"pos": s.tree.pos, "span": s.tree.span, "info": s.tree.info}
    if kind == "attn":
        tree.attn_tree(s.q, s.cache, s.step, s.plan, s.tree, s.scale, s.out)
        return {"out": s.out}
    if kind == "accept":
        a = s.accepted
        tree.tree_accept(s.d_parent, s.d_drafted, s.d_target, s.step, a, given=s.d_given)
        return {"path": a.path, "count": a.count, "token": a.token, "kv_len": a.kv_len}
    if kind == "compact":
        pages.kv_compact(s.caches, s.step, s.d_path, s.d_count)
        return {"kv": s.kv_pool}
    pages.kv_remap(s.d_table, s.d_len, s.d_src, None, s.pool, s.d_head, s.d_next, s.out1)
    pages.kv_copy(s.caches, s.out1)
    pages.kv_remap(s.out1.table, s.out1.kv_len, s.d_back, None, s.pool, s.d_next, s.d_next2,
                   s.out2)
    return _fork_outputs(s)


# ---- what a pass cannot do without ----------------------------------------------------


def work(case):
    """Bytes: every input read once, every output written once; a shared prefix's
    keys and values once a group."""
    past, new, chunk, group = _lengths(case)
    B, T, kind, S = len(past), float(new.sum()), case["kind"], case["page"]
    if kind == "tree":
        # parents in; positions and intervals out; starts, lengths, kinds by request
        return {"bytes": 16.0 * T + 20.0 * B, "flops": 4.0 * T}
    if kind == "accept":
        t = 4.0 if case["dtype"] == "int32" else 8.0
        return {"bytes": (4.0 + 2 * t + 4.0) * T + 28.0 * B, "flops": 2.0 * T}
    row = 4.0 * case["kv_heads"] * case["d"]              # k and v of a key
    if kind == "compact":
        # half of an accepted path's nodes move
        a = np.minimum((case["most"] + 1) / 2.0, (new + 1) // 2)
        moved = float(np.maximum(a - 1, 0).sum()) / 2
        return {"bytes": 2 * row * moved * case["layers"] + 12.0 * T + 8.0 * B, "flops": moved}
    if kind == "fork":
        part, pages, k = past % S, -(-past // S), case["samples"]
        copied = float(part.sum()) * (k - 1) * case["layers"]
        entries = float(pages.sum()) * (1 + k + k + 1)
        return {"bytes": 2 * row * copied + 4.0 * entries + 2 * 12.0 * B * k,
                "flops": float(pages.sum()) * k}
    H, D = case["heads"], case["d"]
    whole = case["prefix"] // S * S
    alone = past + new - np.where(group >= 0, whole, 0)
    keys = float(alone.sum()) + whole * len(set(group[group >= 0].tolist()))
    # a chunk's tokens see half of its new keys, a tree's their ancestors (few)
    seen = np.where(chunk, (new + 1) / 2, np.log2(new + 1))
    pairs = float((new * (past + seen)).sum())
    return {"bytes": row * keys + 4.0 * T * H * D, "flops": 4.0 * D * H * pairs}


# ---- the same by the definitions, in 64 bits and on the host --------------------------


def _ancestors(par, i):
    out = []
    while i >= 0:
        out.append(i)
        i = int(par[i])
    return out[::-1]


def _exact_tree(s):
    pos, span, info = [], [], []
    for b, par in enumerate(s.trees):
        n = len(par)
        kids = [[] for _ in range(n + 1)]                 # the last: the roots
        for i in range(n):
            kids[int(par[i])].append(i)
        first, last, num = [0] * n, [0] * n, 0
        stack = [(i, False) for i in reversed(kids[n])]
        while stack:
            i, done = stack.pop()
            if done:
                last[i] = num - 1
                continue
            first[i] = num
            num += 1
            stack.append((i, True))
            stack.extend((c, False) for c in reversed(kids[i]))
        depth = [0] * n
        for i in range(n):
            depth[i] = depth[int(par[i])] + 1 if par[i] >= 0 else 0
        pos += [int(s.past[b]) + d for d in depth]
        span += list(zip(first, last))
        info.append((int(any(int(p) != i - 1 for i, p in enumerate(par))), 0))
    t = lambda a: _dev(np.array(a, np.int64))
    return {"pos": t(pos), "span": t(span), "info": t(info)}


def _exact_attention(s):
    """Token by token: the cached keys and the token's own path, gathered."""
    q, D, KH = s.q, s.q.shape[2], s.kv_pool.shape[3]
    H = q.shape[1]
    r = H // KH
    kp, vp = s.kv_pool[0, 0], s.kv_pool[0, 1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for b in range(s.B):
        p, n, lo, par = int(s.past[b]), int(s.kv[b]), int(s.starts[b]), s.trees[b]
        m = n - p
        bad = np.ones((m, m), bool)
        for i in range(m):
            if s.chunk[b]:
                bad[i, :i + 1] = False
            else:
                bad[i, _ancestors(par, i)] = False
        bad = torch.from_numpy(bad).to(DEV).repeat_interleave(r, 0)
        idx = torch.arange(n, device=DEV)
        page, off = s.d_table[b].long()[idx // s.page], idx % s.page
        for h in range(KH):
            K, V = kp[page, h, off].double(), vp[page, h, off].double()
            rows = q[lo:lo + m, h * r:(h + 1) * r].double().reshape(m * r, D)
            w = (rows @ K.t()) * s.scale
            w[:, p:] = torch.where(bad, torch.full_like(w[:, p:], -math.inf), w[:, p:])
            out[lo:lo + m, h * r:(h + 1) * r] = (torch.softmax(w, -1) @ V).view(m, r, D)
    return {"out": out}


def _exact_accept(s):
    path, count, token = np.full(s.T, -1, np.int64), [], []
    for b, par in enumerate(s.trees):
        lo, n = int(s.starts[b]), len(par)
        at = list(range(int(s.given[b])))
        while True:
            cur = at[-1]
            fits = [c for c in range(cur + 1, n)
                    if par[c] == cur and s.drafted[lo + c] == s.target[lo + cur]]
            if not fits:
                break
            at.append(fits[0])
        path[lo:lo + len(at)] = at
        count.append(len(at))
        token.append(int(s.target[lo + at[-1]]))
    return {"path": _dev(path), "count": _dev(np.array(count)),
            "token": _dev(np.array(token), DTYPES[s.case["dtype"]]),
            "kv_len": _dev(s.past + np.array(count))}


def _exact_compact(s):
    kv = s.kv_pool.double()
    was = kv.clone()
    place = lambda b, i: (int(s.table[b, (s.past[b] + i) // s.page]), (s.past[b] + i) % s.page)
    for b in range(s.B):
        lo = int(s.starts[b])
        for i in range(int(s.count[b])):
            p0, o0 = place(b, int(s.path[lo + i]))
            p1, o1 = place(b, i)
            kv[:, :, p1, :, o1] = was[:, :, p0, :, o0]
    return {"kv": kv}


def _exact_fork(s):
    """Page by page and request by request."""
    S, kv = s.page, s.kv_pool.double()
    shares, free = s.shares.copy(), s.free_list.copy()
    blank = lambda n: np.zeros((n, s.max_pages), np.int64)

    def remap(table, lens, src, head, out):
        for i, b in enumerate(src):
            for j in range(-(-int(lens[b]) // S)):
                shares[table[b, j]] += 1
        gone = []
        for b in range(len(lens)):
            for j in range(-(-int(lens[b]) // S)):
                shares[table[b, j]] -= 1
        for b in range(len(lens)):
            for j in range(-(-int(lens[b]) // S)):
                if shares[table[b, j]] < 0:
                    shares[table[b, j]] = 0
                    gone.append(table[b, j])
        head -= len(gone)
        free[head:head + len(gone)] = gone
        keep, copies = lens[src], np.full((len(src), 3), -1, np.int64)
        taken = 0
        for i, b in enumerate(src):
            n = -(-int(keep[i]) // S)
            out[i, :n] = table[b, :n]
            p = out[i, n - 1] if n else 0
            if keep[i] % S and shares[p] > 0:
                shares[p] -= 1
                out[i, n - 1] = free[head + taken]
                copies[taken] = p, free[head + taken], keep[i] % S
                taken += 1
        meta = np.zeros(8, np.int64)
        meta[:2] = len(gone), taken
        return out, keep, copies, meta, head + taken

    t1, l1, c1, m1, h1 = remap(s.table, s.kv, s.src, s.lead, blank(s.B * s.k))
    for p, f, n in c1[:m1[1]]:
        kv[:, :, f, :, :n] = kv[:, :, p, :, :n]
    t2, l2, c2, m2, h2 = remap(t1, l1, s.back, h1, blank(s.B))
    d = lambda t, l, c, m, h: {"table": _dev(t), "kv_len": _dev(l), "copies": _dev(c),
                               "meta": _dev(m), "next": _dev(np.array([h]))}
    return {"forked": d(t1, l1, c1, m1, h1), "kept": d(t2, l2, c2, m2, h2),
            "shares": _dev(shares), "free": _dev(free), "kv": kv}


def exact(case, seed):
    if case["kind"] == "attn" and work(case)["flops"] > 1.5e12:
        return None
    s = _inputs(case, seed)
    return {"tree": _exact_tree, "attn": _exact_attention, "accept": _exact_accept,
            "compact": _exact_compact, "fork": _exact_fork}[case["kind"]](s)
