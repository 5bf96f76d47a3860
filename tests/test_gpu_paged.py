"""The operators of a step over a paged cache on the GPU (include/plora_paged.h)
against the float64 oracle: the step's layout bit for bit, the rotation and its
gradient, attention over its row counts, cuts, groups, masks and odd values."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import paged as OP  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2608_05483_amd import paged
    return paged


@pytest.fixture(scope="module")
def P():
    from paper_2608_05483_amd import plora
    return plora


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def f64(t):
    return t.double().cpu().numpy()


# ---- the step's layout ----------------------------------------------------------------


def run_plan(G, past, new, free, head, table, page, T):
    step = G.Step(len(past), T, page, table.shape[1], table=i32(table))
    nxt = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    G.kv_plan(i32(past), i32(new), i32(free), i32([head]), nxt, step)
    torch.cuda.synchronize()
    got = {k: getattr(step, k).cpu().numpy() for k in ("q_start", "kv_len", "pos", "req",
                                                       "slot", "meta", "table")}
    got["next"] = int(nxt.item())
    return got, step


def check_plan(G, past, new, free, head, table, page, T):
    got, _ = run_plan(G, past, new, free, head, table, page, T)
    ref_table = np.array(table)
    ref = OP.kv_plan(past, new, free, head, ref_table, page, T)
    for k, v in ref.items():
        assert np.array_equal(got[k], v), k
    assert np.array_equal(got["table"], ref_table)
    return got


@pytest.mark.parametrize("B,lo,hi,page", [
    (1, 1, 1, 16), (3, 0, 40, 16), (64, 1, 1, 32), (257, 0, 9, 16), (1024, 0, 5, 64),
    (1025, 0, 5, 16),                  # two chunks of requests
    (5000, 0, 3, 256),                 # five
    (7, 100, 700, 16),                 # several work groups of tokens
])
def test_plan_matches(G, B, lo, hi, page):
    rng = np.random.default_rng(B * 7 + page)
    past, new = rng.integers(0, 300, B), rng.integers(lo, hi + 1, B)
    max_pages = int(-(-(past + new).max() // page)) + 2
    table = rng.integers(0, 10 ** 6, (B, max_pages))
    need = int((-(-(past + new) // page) - -(-past // page)).sum())
    free = rng.permutation(need + 9) + 10 ** 6
    T = int(new.sum())
    for pad in (0, 3):                 # rows behind the requests' tokens
        check_plan(G, past, new, free, 5, table, page, T + pad)


def test_plan_leaves_out_what_it_cannot_serve(G):
    page, rng = 16, np.random.default_rng(3)
    table = rng.integers(0, 100, (8, 4))
    past = [0, -1, 60, 5, 0, 3, 16, 2]
    new = [17, 2, 10, -4, 30, 1, 0, 20]
    T = 17 + 2 + 10 + 30 + 1 + 20
    # enough pages; too few for request 4 and then 7; none; head past the list or below it
    for n_free, head in [(40, 0), (3, 0), (40, 37), (0, 0), (5, 9), (5, -2)]:
        check_plan(G, past, new, np.arange(n_free) + 500, head, table, page, T)
    # tokens that pass T, a batch whose lengths overflow, an empty one
    check_plan(G, past, new, np.arange(40), 0, table, page, 25)
    check_plan(G, [0, 2 ** 31 - 1, 1], [2 ** 31 - 1, 2 ** 31 - 1, 3], np.arange(9), 0,
               table[:3], page, 40)
    check_plan(G, [0] * 8, [0] * 8, np.arange(9), 2, table, page, 4)


def test_plan_loop(G):
    """Steps handed on: kv_len and free_next of one are past and free_head of the
    next; no page is given out twice."""
    page, B = 16, 5
    rng = np.random.default_rng(9)
    free = i32(rng.permutation(64))
    table = torch.full((B, 12), -1, dtype=torch.int32, device="cuda")
    past, head = i32(np.zeros(B)), i32([0])
    for n in range(1, 9):
        step = G.Step(B, 5 * n, page, 12, table=table)
        nxt = i32([0])
        G.kv_plan(past, i32([n] * B), free, head, nxt, step)
        past, head = step.kv_len, nxt
    used = table[table >= 0].cpu().numpy()
    assert len(set(used)) == len(used) == int(head.item()) == 5 * 3
    assert (past.cpu().numpy() == 36).all()


# ---- the rotation ---------------------------------------------------------------------


def half_step(dt):
    """Half a step of the type, relative: 8 and 11 significant bits."""
    return 2.0 ** -8 if dt == BF else 2.0 ** -11


def check_rotation(got, ref, x, dt, scale):
    """One rounding (half a step of the type) of a sum of two products whose
    factors are within 2^-22: sinpi and cospi to 2 ulp, an angle to 2^-25 turns."""
    size = np.abs(x).max(-1, keepdims=True) * abs(scale) * 2
    assert (np.abs(got - ref) <= half_step(dt) * np.abs(ref) + 2.0 ** -21 * size + 2.0 ** -25).all()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,rot", [
    (1, 1, 128, 128), (5, 3, 128, 64), (9, 2, 64, 64), (4, 5, 128, 40), (3, 2, 64, 12),
    (3, 2, 10, 6), (2, 3, 6, 6), (7, 2, 128, 0), (2, 1, 256, 256), (1100, 2, 64, 32),
])
def test_rope(G, dt, layout, T, H, D, rot):
    g = torch.Generator(device="cuda").manual_seed(T + D + rot)
    x = torch.randn((T, H, D), device="cuda", generator=g).to(dt)
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 2 ** 31 - 1, T)
    pos[:2] = [0, 131071][:T]
    turns = G.rope_turns(rot, scaling="bands", factor=8.0, original=4096)
    whole = turns.cpu().numpy().view(np.uint64)
    scale = 1.25
    out = torch.zeros_like(x)
    G.rope(x, i32(pos), turns, out, layout=layout, scale=scale)
    ref = OP.rotate(f64(x), pos, whole, layout, scale)
    check_rotation(f64(out), ref, f64(x), dt, scale)
    assert torch.equal(out[..., rot:], x[..., rot:])
    # in place, and the gradient: <R x, y> = <x, R^T y>
    y = x.clone()
    G.rope(y, i32(pos), turns, y, layout=layout, scale=scale)
    assert torch.equal(y, out)
    gx = torch.zeros_like(x)
    G.rope(x, i32(pos), turns, gx, layout=layout, scale=scale, inverse=True)
    check_rotation(f64(gx), OP.rotate(f64(x), pos, whole, layout, scale, True), f64(x), dt, scale)


def test_rope_gradient_by_differences(G):
    """The directional derivative of sum(w * rope(x)) along y, by central
    differences of the oracle in float64, is the product of y with the inverse of w."""
    T, H, D, rot = 6, 2, 64, 32
    rng = np.random.default_rng(1)
    turns = G.rope_turns(rot)
    whole = turns.cpu().numpy().view(np.uint64)
    pos = rng.integers(0, 5000, T)
    x, y = rng.normal(size=(T, H, D)), rng.normal(size=(T, H, D))
    w = torch.from_numpy(rng.normal(size=(T, H, D))).to(BF).cuda()
    for layout in ("half", "interleaved"):
        up = OP.rotate(x + 1e-3 * y, pos, whole, layout, 0.7)
        down = OP.rotate(x - 1e-3 * y, pos, whole, layout, 0.7)
        slope = ((up - down) * f64(w)).sum() / 2e-3
        grad = torch.zeros_like(w)
        G.rope(w, i32(pos), turns, grad, layout=layout, scale=0.7, inverse=True)
        # each of the T H D gradients carries one bf16 rounding
        assert abs((f64(grad) * y).sum() - slope) <= 2.0 ** -8 * (np.abs(f64(grad) * y)).sum()


@pytest.mark.parametrize("dt,layout,T,H,KH,D,rot,page", [
    (BF, "half", 1, 32, 32, 128, 128, 16), (HF, "interleaved", 37, 8, 2, 64, 32, 32),
    (BF, "half", 40, 5, 5, 128, 40, 16), (HF, "half", 1030, 2, 1, 64, 64, 128),
    (BF, "interleaved", 6, 3, 1, 10, 4, 16),
])
def test_rope_append(G, dt, layout, T, H, KH, D, rot, page):
    g = torch.Generator(device="cuda").manual_seed(T)
    mk = lambda *s: torch.randn(s, device="cuda", generator=g).to(dt)
    # strided inputs: q, k, v are slices of one row of projections
    row = mk(T, (H + 2 * KH) * D + 24)
    cut = lambda a, n: row[:, a * D:(a + n) * D].view(T, n, D)
    q, k, v = cut(0, H), cut(H, KH), cut(H + KH, KH)
    rng = np.random.default_rng(T)
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    bad = rng.random(T) < 0.2
    slots[bad] = rng.choice([-1, n_pages * page, 2 ** 40, -2 ** 40], bad.sum())
    pos = rng.integers(0, 9000, T)
    turns = G.rope_turns(rot, base=500000.0)
    whole = turns.cpu().numpy().view(np.uint64)
    # another order of the cache's dimensions: [page][key][head][dim]
    pool = lambda: torch.full((n_pages, page, KH, D), 7.0, dtype=dt, device="cuda")
    cache = G.KVCache(pool().transpose(1, 2), pool().transpose(1, 2))
    out = torch.zeros((T, H, D), dtype=dt, device="cuda")
    G.rope_append(q, k, v, i32(pos), torch.from_numpy(slots).cuda(), turns, cache, out,
                  layout=layout)
    check_rotation(f64(out), OP.rotate(f64(q), pos, whole, layout), f64(q), dt, 1.0)
    rk = OP.rotate(f64(k), pos, whole, layout)
    ck, cv = f64(cache.k), f64(cache.v)
    seen = np.zeros((n_pages, page), bool)
    for t in range(T):
        if 0 <= slots[t] < n_pages * page:
            p, o = divmod(int(slots[t]), page)
            seen[p, o] = True
            check_rotation(ck[p, :, o], rk[t], f64(k)[t], dt, 1.0)
            assert np.array_equal(cv[p, :, o], f64(v)[t])
    untouched = ~seen[:, None, :, None]
    assert (ck[np.broadcast_to(untouched, ck.shape)] == 7).all()
    assert (cv[np.broadcast_to(untouched, cv.shape)] == 7).all()


# ---- attention ------------------------------------------------------------------------


class Batch:
    """A planned step with random caches; groups share pages as a cache of
    prefixes would."""

    def __init__(self, G, P, past, new, H, KH, D=128, page=16, dt=BF, group=None, prefix=(),
                 pad=0, seed=0, max_q=None, order="head"):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        past, new = np.asarray(past), np.asarray(new)
        B, T = len(past), int(new.sum()) + pad
        kv = past + new
        max_pages = int(-(-kv.max() // page)) + 1
        n_pages = int((-(-kv // page)).sum()) + 3
        ids = list(rng.permutation(n_pages))
        table = np.full((B, max_pages), -1)
        lead = {}
        for b in range(B):
            n = 0
            if group is not None and group[b] >= 0:
                n = int(prefix[group[b]]) // page
                if group[b] not in lead:
                    lead[group[b]] = [ids.pop() for _ in range(n)]
                table[b, :n] = lead[group[b]]
            for j in range(n, -(-int(past[b]) // page)):
                table[b, j] = ids.pop()
        self.page, self.KH = page, KH
        mk = lambda *s: torch.randn(s, device="cuda", generator=g).to(dt)
        if order == "head":
            self.cache = G.KVCache(mk(n_pages, KH, page, D), mk(n_pages, KH, page, D))
        else:
            self.cache = G.KVCache(mk(n_pages, page, KH, D).transpose(1, 2),
                                   mk(n_pages, page, KH, D).transpose(1, 2))
        self.q = mk(T, H, D)
        self.out = torch.full((T, H, D), 9.0, dtype=dt, device="cuda")
        self.step = G.Step(B, T, page, max_pages, table=i32(table))
        free = i32(ids)
        G.kv_plan(i32(past), i32(new), free, i32([0]), i32([0]), self.step)
        self.plan = G.AttnPlan(self.step, H, KH, D, max_q=int(new.max()) if max_q is None
                               else max_q, shared=group is not None)
        if group is not None:
            segs = P.Segments(B, len(prefix))
            P.segment(i32(group), segs)
            G.attn_plan(self.step, self.plan, segs, i32(prefix))
        else:
            G.attn_plan(self.step, self.plan)
        self.G = G

    def run(self, scale):
        self.G.attn_paged(self.q, self.cache, self.step, self.plan, scale, self.out)
        torch.cuda.synchronize()
        return f64(self.out)

    def header(self):
        return self.plan.plan[:20].view(torch.int32).tolist()

    def ref(self, scale, rows=None):
        s = self.step
        req = s.req.cpu().numpy()
        if rows is not None:               # these tokens only
            req = np.where(np.isin(np.arange(len(req)), rows), req, -1)
        return OP.attention(f64(self.q), f64(self.cache.k), f64(self.cache.v),
                            s.table.cpu().numpy(), s.q_start.cpu().numpy(),
                            s.kv_len.cpu().numpy(), req, s.pos.cpu().numpy(), self.page, scale)


def check(got, ref, size, dt, keys, vmax=6.0):
    """|error| <= the output's rounding, the weights' rounding to the type (half a
    step each, of sum p |v|), fp32 sums and exponentials (1e-4 of the same), and in
    fp16 the weights below its normal range (half of 2^-24 each, weights summing
    to at least 1 before they are divided)."""
    half = half_step(dt)
    tol = half * np.abs(ref) + (half + 1e-4) * size
    if dt == HF:
        tol = tol + keys * 2.0 ** -25 * vmax + 2.0 ** -24
    assert np.isfinite(got).all()
    worst = (np.abs(got - ref) - tol).max()
    assert worst <= 0, worst


@pytest.mark.parametrize("long", [2100, 4100])
def test_few_tokens_to_merge_among_many(G, P, long):
    """A long prompt, whose rows no partials make, between requests that share a
    prefix, requests of no group and padding, over more tokens than the merge has
    work groups."""
    B = 24
    new = np.where(np.arange(B) % 5 == 4, 3, 1)
    new[B // 2] = long
    group = np.arange(B) % 3 - 1
    group[B // 2] = -1
    b = Batch(G, P, [96 + 7 * i for i in range(B)], new, 4, 2, 64, group=group, prefix=[64, 96],
              pad=133, seed=long)
    got = b.run(0.125)
    start = b.step.q_start.cpu().numpy()
    lo, hi = start[B // 2], start[B // 2 + 1]
    rows = np.r_[0:lo + 3, lo + 2040:lo + 2060, hi - 3:len(got)]
    ref, size = b.ref(0.125, rows)
    check(got[rows], ref[rows], size[rows], BF, 6000)
    assert (got[start[-1]:] == 0).all()


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("new", [1, 40])
def test_many_keys_of_little_weight_fp16(G, P, D, new):
    """Every 64th key has the weight 1 and a value of zero; what is left of the
    output is that of the others, whose weights of 2^-25.5 are below half of fp16's
    smallest number.  A weight may be off by half of that 2^8 lower (2^-33)."""
    b = Batch(G, P, [700], [new], 2, 1, D, page=32, dt=HF)
    scale = 1.0 / 16
    b.q.fill_(1.0)
    sink = 25.5 * math.log(2.0) / (D * scale)
    table = b.step.table.cpu().numpy()[0]
    off = torch.arange(32, device="cuda")
    for j in range(-(-(700 + new) // 32)):
        first = ((j * 32 + off) % 64 == 0)[None, :, None]
        k, v = b.cache.k[int(table[j])], b.cache.v[int(table[j])]
        k.copy_(torch.where(first, sink, 0.0).expand_as(k))
        v.copy_(torch.where(first, 0.0, 30000.0).expand_as(v))
    got = b.run(scale)
    ref, size = b.ref(scale)
    assert ref.min() > 0.02
    tol = half_step(HF) * np.abs(ref) + (half_step(HF) + 1e-4) * size + 64 * 2.0 ** -33 * 30000
    assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 128), (BF, 64), (HF, 64)])
@pytest.mark.parametrize("H,KH", [(4, 4), (8, 1), (16, 1), (6, 2), (20, 1), (40, 2)])
def test_decode(G, P, dt, D, H, KH):
    """One token a request: 1, 3, 8, 16 rows a key head (one tile), 20 (more)."""
    past = [0, 1, 14, 15, 16, 31, 32, 127, 128, 300, 511, 1000]
    b = Batch(G, P, past, [1] * len(past), H, KH, D, dt=dt, seed=H + D)
    got = b.run(D ** -0.5)
    check(got, *b.ref(D ** -0.5), dt, 1000)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("order", ["head", "key"])
def test_few_tokens_a_request(G, P, page, order):
    """0 to 9 tokens of 2 heads a key head, behind caches of odd lengths: tiles of
    up to 16 rows and of more, causal inside the new tokens; padding rows."""
    past, new = [0, 5, 37, 64, 100, 0, 700, 333, 15], [3, 1, 9, 0, 7, 1, 8, 2, 4]
    b = Batch(G, P, past, new, 4, 2, page=page, pad=5, order=order)
    got = b.run(0.2)
    ref, size = b.ref(0.2)
    check(got, ref, size, BF, 800)
    assert (got[-5:] == 0).all()


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("past,new,H,KH", [
    ([0], [1], 2, 1), ([0], [33], 3, 1), ([0, 0, 70], [129, 64, 200], 2, 2),
    ([0], [300], 8, 1), ([500, 16], [127, 1], 2, 1),
])
def test_prompts(G, P, dt, D, past, new, H, KH):
    b = Batch(G, P, past, new, H, KH, D, dt=dt, seed=sum(new))
    got = b.run(D ** -0.5)
    check(got, *b.ref(D ** -0.5), dt, 700)


@pytest.mark.parametrize("H,KH,new", [(4, 1, 1), (32, 2, 1), (3, 1, 40)])
def test_long_cache_is_cut(G, P, H, KH, new):
    """Few rows, many keys: several pieces, joined."""
    b = Batch(G, P, [9000, 7000], [new, new], H, KH, seed=H)
    got = b.run(0.09)
    assert b.header()[2] > 0
    check(got, *b.ref(0.09), BF, 9000)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("H,KH,hi", [(2, 2, 1), (8, 1, 1), (4, 1, 6), (16, 1, 30)])
def test_shared_prefixes(G, P, dt, D, H, KH, hi):
    """Groups of 1, 2, 5 and more members with prefixes of 0, less than a page and
    several pages; requests of no group; members with many rows, which attend
    alone.  The result is that of unshared attention over the same pages."""
    rng = np.random.default_rng(H + hi)
    B = 24
    group = rng.choice([-1, 0, 1, 2, 3, 4], B)
    group[:3] = [5, 1, 1]                         # group 5 has one member
    prefix = np.array([0, 200, 7, 64, 1025, 48])
    past = rng.integers(0, 90, B) + np.where(group >= 0, prefix[group], 0)
    new = rng.integers(1, hi + 1, B)
    if hi > 1:
        new[4] = 0
    b = Batch(G, P, past, new, H, KH, D, dt=dt, group=group, prefix=prefix, seed=hi)
    got = b.run(0.1)
    check(got, *b.ref(0.1), dt, 1200)
    # without groups: the same within both roundings
    c = G.AttnPlan(b.step, H, KH, D, max_q=int(new.max()))
    G.attn_plan(b.step, c)
    b.plan = c
    check(b.run(0.1), *b.ref(0.1), dt, 1200)


@pytest.mark.parametrize("share", [False, True])
def test_many_requests(G, P, share):
    """More requests than the plan's kernel keeps in LDS, and more than it takes at a
    time; 70 groups and some requests in none."""
    rng = np.random.default_rng(5)
    n, prefix = 1300, rng.integers(0, 80, 70)
    group = rng.integers(-1, 70, n)
    past = rng.integers(0, 100, n) + np.where(group >= 0, prefix[group], 0)
    new = np.where(rng.random(n) < 0.02, 20, rng.integers(0, 3, n))
    b = Batch(G, P, past, new, 2, 1, 64, group=group if share else None,
              prefix=prefix if share else (), seed=5)
    check(b.run(0.125), *b.ref(0.125), BF, 200)


def test_a_request_inside_its_prefix_does_not_share(G, P):
    """A request that is still writing the prefix attends alone; ids outside the
    groups and negative prefixes share nothing."""
    group = np.array([0, 0, 0, 1, 1, 7, 2, 2])
    prefix = np.array([64, 64, -5])
    past = np.array([64, 80, 64, 70, 70, 70, 20, 20])
    b = Batch(G, P, past, [2] * 8, 4, 2, group=np.where(group > 2, -1, group),
              prefix=np.maximum(prefix, 0))
    short = b.step.kv_len.clone()
    segs = P.Segments(8, 3)
    P.segment(i32(group), segs)
    G.attn_plan(b.step, b.plan, segs, i32(np.array([65, 64, -5])))
    assert torch.equal(short, b.step.kv_len)
    check(b.run(0.1), *b.ref(0.1), BF, 100)
    # the prefix is longer than what the requests held: nothing to share
    G.attn_plan(b.step, b.plan, segs, i32(np.array([2 ** 31 - 1, 4000, 96])))
    check(b.run(0.1), *b.ref(0.1), BF, 100)


@pytest.mark.parametrize("H,KH,new", [(2, 1, 5), (4, 1, 50)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_masked_values_have_no_part(G, P, H, KH, new, value):
    """Infinities and NaN in keys and values that a row does not see: those of
    later tokens, of the page behind the last key, and of pages of others."""
    past = [20, 100]
    b = Batch(G, P, past, [new, new], H, KH)
    s = b.step
    ref, size = b.ref(0.3)
    table = s.table.cpu().numpy()
    slot = s.slot.cpu().numpy()
    used = set()
    for r in range(2):
        for j in range(past[r] + new):
            used.add(int(table[r, j // 16]) * 16 + j % 16)
    flat_k = b.cache.k.transpose(1, 2).clone()
    flat_v = b.cache.v.transpose(1, 2).clone()
    last = [new - 1, 2 * new - 1]
    for i in range(flat_k.shape[0] * 16):
        if i not in used or i in (slot[last[0]], slot[last[1]]):
            flat_k[i // 16, i % 16] = value
            flat_v[i // 16, i % 16] = value
    b.cache.k.copy_(flat_k.transpose(1, 2))
    b.cache.v.copy_(flat_v.transpose(1, 2))
    got = b.run(0.3)
    seen = [t for t in range(2 * new) if t not in last]
    check(got[seen], ref[seen], size[seen], BF, 200)
    # the rows that do see them are not finite numbers
    assert not np.isfinite(got[last]).all()


def test_infinite_values_that_are_seen(G, P):
    """A seen infinity in one dimension of v gives that dimension's infinity and
    leaves the others."""
    for H, new in ((2, 2), (8, 20)):
        b = Batch(G, P, [40], [new], H, 1)
        ref, size = b.ref(0.2)
        page = int(b.step.table[0, 0])
        b.cache.v[page, 0, 3, 5] = math.inf
        b.cache.v[page, 0, 4, 9] = -math.inf
        got = b.run(0.2)
        assert (got[..., 5] == math.inf).all() and (got[..., 9] == -math.inf).all()
        rest = [d for d in range(128) if d not in (5, 9)]
        check(got[..., rest], ref[..., rest], size[..., rest], BF, 60)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 4.0])
def test_scales(G, P, scale):
    """Flat weights, reversed ones, and scores far past exp's range."""
    for H, new in ((4, 1), (4, 30)):
        b = Batch(G, P, [200, 3], [new, new], H, 2, seed=4)
        check(b.run(scale), *b.ref(scale), BF, 250)


def test_rising_scores(G, P):
    """Keys whose scores rise along the cache by far more than the slack under
    which the output is not rescaled, and by less."""
    for step in (0.5, 0.05, -0.5):
        for H, new in ((2, 1), (4, 40)):
            b = Batch(G, P, [700], [new], H, 1, seed=5)
            b.q.fill_(0.25)
            n = 700 + new
            table = b.step.table[0].long()
            for j in range(n):
                b.cache.k[table[j // 16], :, j % 16] = (j - n / 2) * step / 32
            check(b.run(0.25), *b.ref(0.25), BF, 800)


def test_more_tokens_than_stated_and_left_out_requests_get_zeros(G, P):
    b = Batch(G, P, [10, 10, 10], [2, 9, 3], 4, 2, max_q=4)
    got = b.run(0.2)
    ref, size = b.ref(0.2)
    ref[2:11], size[2:11] = 0, 0
    check(got, ref, size, BF, 20)
    assert (got[2:11] == 0).all()


def test_pages_outside_the_pool_read_as_zeros(G, P):
    b = Batch(G, P, [100, 60], [1, 20], 4, 2)
    table = b.step.table
    table[0, 2], table[1, 1] = 10 ** 6, -3
    got = b.run(0.2)
    zero = b.cache.n_pages
    pad = lambda t: torch.cat([t, torch.zeros_like(t[:1])])
    b.cache.k, b.cache.v = pad(b.cache.k), pad(b.cache.v)
    table[0, 2], table[1, 1] = zero, zero
    check(got, *b.ref(0.2), BF, 120)


def test_offsets_past_32_bits(G, P):
    """A pool of more than 2^32 bytes and 2^31 elements: the last pages."""
    KH, D, page = 8, 128, 64
    n_pages = (2 ** 31 + 2 ** 29) // (KH * D * page) + 7
    k = torch.zeros((n_pages, KH, page, D), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    k[-4:].normal_(), v[-4:].normal_()
    cache = G.KVCache(k, v)
    B, new = 2, [1, 20]
    table = np.array([[n_pages - 1, n_pages - 2], [n_pages - 3, n_pages - 4]])
    step = G.Step(B, 21, page, 2, table=i32(table))
    G.kv_plan(i32([100, 90]), i32(new), i32([]), i32([0]), i32([0]), step)
    q = torch.randn((21, 16, D), device="cuda").to(BF)
    kk, vv = torch.randn((21, KH, D), device="cuda").to(BF), torch.randn((21, KH, D), device="cuda").to(BF)
    out = torch.zeros_like(q)
    plan = G.AttnPlan(step, 16, KH, D, max_q=20)
    G.attn_plan(step, plan)
    turns = G.rope_turns(D)
    G.run_layers(step, plan, [(q, kk, vv, cache, out)], turns, 0.1)
    torch.cuda.synchronize()
    small = lambda t: f64(t[-4:])
    ref, size = OP.attention(f64(q), small(k), small(v), table - (n_pages - 4), None, None,
                             step.req.cpu().numpy(), step.pos.cpu().numpy(), page, 0.1)
    check(f64(out), ref, size, BF, 120)
    slot = step.slot.cpu().numpy()
    at = k.view(n_pages, KH, page, D)[n_pages - 2, :, 100 - 64]
    assert slot[0] == (n_pages - 2) * page + 36
    whole = turns.cpu().numpy().view(np.uint64)
    check_rotation(f64(at)[None], OP.rotate(f64(kk[:1]), [100], whole, "half"), f64(kk[:1]), BF, 1)


def test_strided_queries_and_outputs_on_another_stream(G, P):
    """q and out as slices of wider rows; a stream of the caller's; nothing around
    the output is written; the same bits every time."""
    b = Batch(G, P, [50, 700, 3], [1, 4, 30], 4, 2)
    want = b.run(0.1)
    T = b.q.shape[0]
    wide_q = torch.full((T, 6, 160), 3.0, dtype=BF, device="cuda")
    wide_o = torch.full((T, 6, 160), 5.0, dtype=BF, device="cuda")
    q, out = wide_q[:, 1:5, 16:144], wide_o[:, 1:5, 16:144]
    q.copy_(b.q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        G.attn_paged(q, b.cache, b.step, b.plan, 0.1, out, stream=s)
        s.synchronize()
        assert np.array_equal(f64(out), want)
    keep = wide_o.clone()
    keep[:, 1:5, 16:144] = 5.0
    assert (keep == 5.0).all()


def test_a_step_in_a_graph(G, P):
    """The whole step captured: plan, groups, attention's plan, two layers; replayed
    with other lengths in the same buffers, against eager calls."""
    B, page, KH, H, D = 6, 16, 2, 8, 128
    group, prefix = i32([0, 0, 0, 1, 1, -1]), i32([48, 20])
    n_pages, max_pages = 80, 8
    rng = np.random.default_rng(2)
    perm = rng.permutation(n_pages)
    table0 = np.full((B, max_pages), -1)
    table0[:3, :3], table0[3:5, :1] = perm[:3], perm[3:4]
    for r in range(B):
        for j in range(max_pages):
            if table0[r, j] < 0:
                table0[r, j] = perm[4 + r * max_pages + j]
    mk = lambda *s: torch.randn(s, device="cuda").to(BF)
    layers = [[mk(B, H, D), mk(B, KH, D), mk(B, KH, D),
               G.KVCache(mk(n_pages, KH, page, D), mk(n_pages, KH, page, D)),
               torch.zeros((B, H, D), dtype=BF, device="cuda")] for _ in range(2)]
    keep_q = [x[0].clone() for x in layers]
    past, new = i32([60, 70, 48, 30, 44, 9]), i32([1] * B)
    step = G.Step(B, B, page, max_pages, table=i32(table0))
    plan = G.AttnPlan(step, H, KH, D, max_q=1, shared=True)
    segs = P.Segments(B, 2)
    turns, free, head, nxt = G.rope_turns(D), i32([]), i32([0]), i32([0])

    def call():
        G.kv_plan(past, new, free, head, nxt, step)
        P.segment(group, segs)
        G.attn_plan(step, plan, segs, prefix)
        G.run_layers(step, plan, layers, turns, 0.1)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    pool0 = [(x[3].k.clone(), x[3].v.clone()) for x in layers]

    def reset():
        for x, q, (k, v) in zip(layers, keep_q, pool0):
            x[0].copy_(q), x[3].k.copy_(k), x[3].v.copy_(v), x[4].zero_()

    for lens in ([60, 70, 48, 30, 44, 9], [100, 50, 49, 21, 90, 0], [48, 48, 47, 16, 15, 111]):
        past.copy_(i32(lens))
        new.copy_(i32([1] * 5 + [0 if lens[5] == 0 else 1]))
        reset()
        call()
        want = [x[4].clone() for x in layers]
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip(layers, want):
            assert torch.equal(x[4], w)
