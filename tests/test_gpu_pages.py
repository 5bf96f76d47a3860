"""Upkeep of a paged cache on the GPU (include/plora_pages.h) against the oracle, bit
for bit: remaps alone and over many steps, copies and compaction over types, strides
and layers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import pages as OG  # noqa: E402
from test_gpu_paged import BF, HF, G, P, i32  # noqa: E402, F401


@pytest.fixture(scope="module")
def K():
    from paper_2608_05483_amd import pages
    return pages


def arr(t):
    return t.cpu().numpy()


def check_remap(K, table, kv_len, src, keep, page, shares, free, head, new_max=None, fill=-5):
    """One call against the oracle; returns the new state."""
    N, most = len(src), np.asarray(table).shape[1] if new_max is None else new_max
    pool = K.PagePool(i32(shares), i32(free))
    out = K.Remap(len(kv_len), N, page, most,
                  table=torch.full((N, most), fill, dtype=torch.int32, device="cuda"))
    nxt = i32([-7])
    d_table, d_len = i32(table), i32(kv_len)
    K.kv_remap(d_table, d_len, i32(src), None if keep is None else i32(keep), pool, i32([head]),
               nxt, out)
    torch.cuda.synchronize()
    r_shares, r_free = np.array(shares), np.array(free)
    r_table = np.full((N, most), fill)
    ref = OG.remap(np.asarray(table), kv_len, src, keep, page, r_shares, r_free, head, r_table)
    assert np.array_equal(arr(out.kv_len), ref["kv_len"])
    assert np.array_equal(arr(out.meta), ref["meta"])
    assert int(nxt.item()) == ref["next"]
    assert np.array_equal(arr(out.copies).reshape(-1, 3), ref["copies"])
    assert np.array_equal(arr(out.table), r_table)
    assert np.array_equal(arr(pool.shares), r_shares)
    assert np.array_equal(arr(pool.free_pages), r_free)
    assert np.array_equal(arr(d_table), table) and np.array_equal(arr(d_len), kv_len)
    return r_table, np.array(ref["kv_len"]), r_shares, r_free, ref["next"], ref


def fresh(B, most, page, rng, lead=6, spare=40, lens=None):
    """B requests with pages of their own."""
    lens = rng.integers(0, most * page + 1, B) if lens is None else np.asarray(lens)
    n = int((-(-lens // page)).sum())
    ids = rng.permutation(n + spare)
    table, at = np.full((B, most), -9), 0
    for b in range(B):
        k = -(-int(lens[b]) // page)
        table[b, :k] = ids[at:at + k]
        at += k
    free = np.concatenate([np.full(lead, -3), ids[at:]])
    return table, lens, np.zeros(n + spare, np.int64), free, lead


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("B,most", [(1, 1), (1, 9), (5, 4), (64, 7), (300, 3), (1100, 5)])
def test_fork_each(K, page, B, most):
    """Each request continued 0 to 4 times, in any order, lengths of their own."""
    rng = np.random.default_rng(B + most + page)
    table, lens, shares, free, head = fresh(B, most, page, rng, spare=4 * B + 8, lead=B * most + 3)
    src = rng.permutation(np.repeat(np.arange(B), rng.integers(0, 5, B)))
    if len(src) == 0:
        src = np.array([0, 0])
    check_remap(K, table, lens, src, None, page, shares, free, head)
    keep = rng.integers(-3, most * page + 5, len(src))
    check_remap(K, table, lens, src, keep, page, shares, free, head)
    check_remap(K, table, lens, src, keep, page, shares, free, head, new_max=max(1, most // 2))


def test_steps_keep_count_of_every_page(K):
    """Many remaps one after the other: forks, cuts, ends, new tokens in between.  Every
    page is at all times free, or held as often as its count says."""
    rng, page, most, n_pages = np.random.default_rng(3), 16, 6, 400
    free = rng.permutation(n_pages)
    shares, head = np.zeros(n_pages, np.int64), 0
    table, lens = np.full((8, most), -1), np.zeros(8, np.int64)
    for step in range(40):
        # new tokens, as a step's layout gives them pages
        for b in range(len(lens)):
            n = min(int(rng.integers(0, 20)), most * page - int(lens[b]))
            for j in range(-(-int(lens[b]) // page), -(-(int(lens[b]) + n) // page)):
                table[b, j] = free[head]
                head += 1
            lens[b] += n
        N = int(rng.integers(1, 14))
        src = rng.integers(-1, len(lens) + 1, N)
        keep = None if step % 3 == 0 else rng.integers(0, most * page + 1, N)
        table, lens, shares, free, head, ref = check_remap(K, table, lens, src, keep, page, shares,
                                                           free, head)
        assert ref["meta"][2] == ref["meta"][3] == 0
        held = np.zeros(n_pages, np.int64)
        for b in range(len(lens)):
            held[table[b, :-(-int(lens[b]) // page)]] += 1
            if lens[b] % page:               # nobody else writes behind its keys
                assert held[table[b, lens[b] // page]] >= 1
        assert np.array_equal(shares, np.maximum(held - 1, 0))
        listed = free[head:]
        assert len(set(listed)) == len(listed) == n_pages - (held > 0).sum()
        assert (held[listed] == 0).all()
        for b in range(len(lens)):
            if lens[b] % page:
                assert held[table[b, lens[b] // page]] == 1


def test_pages_held_by_others(K):
    """Prompts that requests share with each other and with somebody outside; forks
    that end in the middle of a shared page."""
    rng, page = np.random.default_rng(1), 16
    table = np.array([[10, 11, 1], [10, 11, 2], [10, 11, 3], [4, 5, 6]])
    shares = np.zeros(20, np.int64)
    shares[[10, 11]] = 3                          # three requests and the prompt's owner
    lens, free = np.array([40, 48, 33, 48]), np.concatenate([np.full(12, -1), np.arange(12, 20)])
    for src, keep in [([0, 1, 2, 3], None), ([3], None), ([], None), ([0, 0, 1], [20, 40, 20]),
                      ([0, 1, 2], [20, 20, 20]), ([3, 3, 3], [48, 32, 17]),
                      ([3, 3, 3], [5, 5, 48]), ([0, 0], [16, 32]), ([1, 3, -1, 9, 3], None)]:
        src = np.array(src, np.int64)
        check_remap(K, table, lens, src, keep, page, shares, free, 12)
    out = shares.copy()
    out[[10, 11]] = 2                             # the owner is gone: the last one frees them
    check_remap(K, table, lens, np.array([3]), None, page, out, free, 12)


def test_a_list_too_short(K):
    """No page to give, no room for what comes free, heads outside the list."""
    rng, page = np.random.default_rng(5), 16
    table, lens, shares, _, _ = fresh(6, 4, page, rng, lens=[40, 17, 64, 5, 50, 33], spare=10)
    P = len(shares)
    src = np.array([0, 0, 0, 1, 1, 2, 2, 4, 4, 4])
    for n_free, head in [(0, 0), (1, 0), (3, 1), (3, 3), (40, 2), (5, -1), (5, 6), (4, 2 ** 31 - 1),
                         (4, -2 ** 31)]:
        check_remap(K, table, lens, src, None, page, shares, np.arange(n_free) % P, head)
        check_remap(K, table, lens, src[:1], None, page, shares, np.arange(n_free) % P, head)
    # what comes free is what is given out
    check_remap(K, table, lens, np.array([2, 0, 0]), [64, 40, 39], page, shares,
                np.full(9, 3), 9)


def test_odd_lengths_and_pages(K):
    rng, page = np.random.default_rng(7), 16
    table = rng.permutation(24).reshape(6, 4)
    table[0, 1], table[2, 0], table[4, 3], table[5, 2] = -1, 24, 2 ** 31 - 1, -2 ** 31
    lens = np.array([40, -5, 7, 2 ** 31 - 1, 64, 48])
    free = np.concatenate([np.full(24, -1), np.arange(24)])
    shares = np.zeros(24, np.int64)
    for src in ([0, 0, 1, 2, 2, 3, 4, 4, 5, 5], [5, 4, 3, 2, 1, 0], [2 ** 31 - 1, -2 ** 31, 6, -1]):
        check_remap(K, table, lens, np.array(src), None, page, shares, free, 24)
        check_remap(K, table, lens, np.array(src), np.full(len(src), 20), page, shares, free, 24)
    check_remap(K, table[:0], lens[:0], np.array([0, -1]), None, page, shares, free, 24)
    check_remap(K, table, lens, np.array([], np.int64), None, page, shares, free, 24)
    check_remap(K, table[:, :0], lens, np.array([0, 1]), None, page, shares, free, 24)
    check_remap(K, table[:0], lens[:0], np.array([], np.int64), None, page, shares, free, 24)
    check_remap(K, table, np.full(6, 16), np.array([1, 1]), None, page, shares[:0], free[:0], 0)


def test_many_pages_come_free(K):
    """More entries than are looked at together, over more requests than that."""
    rng = np.random.default_rng(11)
    for B, most in ((40, 200), (1500, 4), (2100, 2), (70, 300), (1300, 60)):
        table, lens, shares, free, head = fresh(B, most, 16, rng, lead=B * most, spare=3000)
        check_remap(K, table, lens, rng.integers(0, B, B // 3), None, 16, shares, free, head)


@pytest.mark.parametrize("grow", [False, True])
def test_long_shared_rows_are_dropped(K, grow):
    """Continuations of long requests, most of which end in the next remap while others go
    on with their pages; some pages are dropped by several and held by none."""
    rng, page, most, B = np.random.default_rng(17), 16, 700, 24
    lens = rng.integers(page * 300, page * most, B)
    table, lens, shares, free, head = fresh(B, most, page, rng, lens=lens, spare=400,
                                            lead=B * most)
    src = np.repeat(np.arange(B), 5)
    table, lens, shares, free, head, _ = check_remap(K, table, lens, src, None, page, shares, free,
                                                     head)
    on = rng.choice(len(src), 160 if grow else 20)
    keep = rng.integers(0, page * most, len(on))
    check_remap(K, table, lens, on, keep, page, shares, free, head)


# ---- copies and compaction ------------------------------------------------------------


def caches(G, K, layers, n_pages, KH, page, D, dt, form, seed=0):
    """Caches of several layouts and alignments; all elements, padding too, are random."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out, whole = [], []
    for _ in range(2 * layers):
        mk = lambda *s: torch.randn(s, device="cuda", generator=g).to(dt)
        if form == "plain":
            w = mk(n_pages, KH, page, D)
            x = w
        elif form == "key":
            w = mk(n_pages, page, KH, D)
            x = w.transpose(1, 2)
        else:                                 # rows that begin at odd multiples of 2 bytes
            w = mk(n_pages, KH, page, D + form + 1)
            x = w[..., form:form + D]
        whole.append(w)
        out.append(x)
    cs = [G.KVCache(out[2 * i], out[2 * i + 1]) for i in range(layers)]
    return K.Caches(cs), out, whole


FORMS = [("plain", 128), ("key", 64), ("plain", 80), ("plain", 36), ("plain", 10), (7, 64), (2, 32),
         (1, 24), (1, 7), ("key", 6)]


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("form,D", FORMS)
@pytest.mark.parametrize("layers,KH", [(1, 1), (3, 5), (66, 2)])
def test_copy(G, K, dt, form, D, layers, KH):
    page, n_pages = 16, 24
    cs, xs, ws = caches(G, K, layers, n_pages, KH, page, D, dt, form)
    rng = np.random.default_rng(D + layers)
    ids = rng.permutation(n_pages)
    rows = [(ids[0], ids[1], 16), (ids[2], ids[3], 1), (ids[4], ids[5], 0), (ids[6], ids[7], -4),
            (ids[6], ids[8], 40), (ids[6], ids[9], 7), (-1, ids[10], 5), (ids[11], -1, 5),
            (n_pages, ids[12], 5), (ids[11], 2 ** 31 - 1, 5), (ids[13], ids[14], 9)]
    out = K.Remap(3, len(rows), page, 2)
    out.copies.copy_(i32(np.array(rows)))
    want = [w.double().cpu().numpy() for w in ws]
    for n in (0, 10):                         # (the last row is behind the count)
        out.meta[1] = n
        K.kv_copy(cs, out)
    torch.cuda.synchronize()
    for w, x, y in zip(ws, xs, want):
        view = torch.from_numpy(y).as_strided(x.shape, x.stride(), x.storage_offset()).numpy()
        OG.copy(view, rows, 10)
        assert np.array_equal(w.double().cpu().numpy(), y)
    out.meta[1] = 2 ** 31 - 1                 # more than there are rows
    K.kv_copy(cs, out)
    for x in xs[:2]:
        assert torch.equal(x[int(ids[14]), :, :9], x[int(ids[13]), :, :9])


def stepped(G, past, new, page, n_pages, rng):
    B = len(past)
    kv = np.asarray(past) + np.asarray(new)
    most = int(-(-kv.max() // page))
    ids = rng.permutation(n_pages)[:B * most].reshape(B, most)
    step = G.Step(B, int(np.sum(new)) + 2, page, most, table=i32(ids))
    held = -(-np.asarray(past) // page)
    free = np.concatenate([ids[b, held[b]:-(-kv[b] // page)] for b in range(B)])
    G.kv_plan(i32(past), i32(new), i32(free), i32([0]), i32([0]), step)
    return step


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("form,D", FORMS)
@pytest.mark.parametrize("layers,KH", [(1, 1), (2, 40), (65, 3)])
def test_compact(G, K, dt, form, D, layers, KH):
    """Paths that stay, that move keys onto places that others moved from, whole
    chains, numbers outside the request, counts outside its tokens."""
    page, n_pages = 16, 40
    rng = np.random.default_rng(D + KH)
    cs, xs, ws = caches(G, K, layers, n_pages, KH, page, D, dt, form, seed=2)
    past, new = [0, 5, 30, 17, 60, 3, 9], [9, 1, 33, 0, 8, 20, 12]
    step = stepped(G, past, new, page, n_pages, rng)
    path, count = [], []
    for b, n in enumerate(new):
        a = int(rng.integers(0, n + 1))
        p = np.full(n, -1)
        p[:a] = np.sort(rng.permutation(n)[:a])
        path.append(p)
        count.append(a)
    path[2] = np.where(np.arange(33) < 32, np.arange(33) + 1, -1)   # each key one down
    count[2] = 33
    path[4], count[4] = np.array([-1, 8, 3, 2 ** 31 - 1, 4, -9, 7, 7]), 8
    path[5], count[5] = np.arange(20), 99
    count[6] = -3
    path = np.concatenate(path + [[0, 0]])
    want = [w.double().cpu().numpy() for w in ws]
    K.kv_compact(cs, step, i32(path), i32(count))
    torch.cuda.synchronize()
    s = {k: arr(getattr(step, k)) for k in ("q_start", "req", "slot")}
    for w, x, y in zip(ws, xs, want):
        view = torch.from_numpy(y).as_strided(x.shape, x.stride(), x.storage_offset()).numpy()
        OG.compact(view, s["q_start"], s["req"], s["slot"], path, count)
        assert np.array_equal(w.double().cpu().numpy(), y)


@pytest.mark.parametrize("down", [1, 3, 64, 100])
def test_compact_of_long_paths(G, K, down):
    """More moves than are looked up at once, each onto a place that another is read
    from later."""
    rng = np.random.default_rng(down)
    cs, xs, ws = caches(G, K, 2, 40, 3, 16, 64, BF, "plain")
    new = [210, 66]
    step = stepped(G, [7, 30], new, 16, 40, rng)
    path, count = np.full(sum(new) + 2, -1), []
    for b, n in enumerate(new):
        lo, a = sum(new[:b]), max(n - down, 0)
        path[lo:lo + a] = np.arange(a) + down
        count.append(a)
    want = [w.double().cpu().numpy() for w in ws]
    K.kv_compact(cs, step, i32(path), i32(count))
    s = {k: arr(getattr(step, k)) for k in ("q_start", "req", "slot")}
    for w, y in zip(ws, want):
        OG.compact(y, s["q_start"], s["req"], s["slot"], path, count)
        assert np.array_equal(w.double().cpu().numpy(), y)


def test_compact_with_slots_outside_the_pool(G, K):
    rng = np.random.default_rng(0)
    cs, xs, ws = caches(G, K, 2, 8, 2, 16, 64, BF, "plain")
    step = stepped(G, [4, 0], [6, 5], 16, 8, rng)
    step.slot[1], step.slot[4], step.slot[8] = -1, 8 * 16, 2 ** 62
    path, count = np.array([0, 2, 3, 4, 5, -1, 1, 2, 3, 4, -1, 0, 0]), [5, 4]
    want = [w.double().cpu().numpy() for w in ws]
    K.kv_compact(cs, step, i32(path), i32(count))
    s = {k: arr(getattr(step, k)) for k in ("q_start", "req", "slot")}
    for w, y in zip(ws, want):
        OG.compact(y, s["q_start"], s["req"], s["slot"], path, count)
        assert np.array_equal(w.double().cpu().numpy(), y)


def test_offsets_past_32_bits(G, K):
    """A pool of more than 2^32 bytes: its last pages copied and compacted; and keys
    that lie 2^31 elements apart in a page."""
    KH, D, page = 8, 128, 64
    n_pages = (2 ** 31 + 2 ** 29) // (KH * D * page) + 7
    k = torch.zeros((n_pages, KH, page, D), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    k[-4:].normal_(), v[-4:].normal_()
    cs = K.Caches([G.KVCache(k, v)])
    out = K.Remap(1, 1, page, 1)
    out.copies.copy_(i32([[n_pages - 1, n_pages - 5, 50]]))
    out.meta[1] = 1
    K.kv_copy(cs, out)
    for x in (k, v):
        assert torch.equal(x[n_pages - 5, :, :50], x[n_pages - 1, :, :50])
        assert (x[n_pages - 5, :, 50:] == 0).all() and (x[n_pages - 6] == 0).all()
    step = G.Step(1, 9, page, 2, table=i32([[n_pages - 2, n_pages - 3]]))
    G.kv_plan(i32([60]), i32([9]), i32([n_pages - 3]), i32([0]), i32([0]), step)
    moved = [x[n_pages - 3, :, 3].clone() for x in (k, v)]
    K.kv_compact(cs, step, i32([0, 7] + [-1] * 7), i32([2]))
    for x, m in zip((k, v), moved):
        assert torch.equal(x[n_pages - 2, :, 61], m)
    del k, v, cs
    torch.cuda.empty_cache()
    stride = 40 << 20
    size = 63 * stride + 2 * 128
    x = [torch.empty(size, dtype=BF, device="cuda").as_strided((2, 1, 64, 128),
                                                               (128, 128, stride, 1))
         for _ in range(2)]
    for y in x:
        y.normal_()
    cs = K.Caches([G.KVCache(*x)])
    out.copies.copy_(i32([[0, 1, 64]]))
    K.kv_copy(cs, out)
    assert torch.equal(x[0][0], x[0][1]) and torch.equal(x[1][0], x[1][1])


def test_a_loop_in_a_graph(G, K):
    """Fork, copy, drop, captured and replayed with other lengths and continuations,
    against eager calls on the same state."""
    B, N, page, most = 5, 12, 16, 6
    rng = np.random.default_rng(4)
    table, _, shares, free, head = fresh(B, most, page, rng, lens=[most * page] * B, spare=40,
                                         lead=B * most + N)
    cs, xs, _ = caches(G, K, 3, len(shares), 2, page, 64, BF, "plain")
    pool = K.PagePool(i32(shares), i32(free))
    a, b = K.Remap(B, N, page, most), K.Remap(N, B, page, most)
    d_table, lens, src, back = i32(table), i32([0] * B), i32([0] * N), i32([0] * B)
    h, h1, h2 = i32([head]), i32([0]), i32([0])

    def call():
        K.kv_remap(d_table, lens, src, None, pool, h, h1, a)
        K.kv_copy(cs, a)
        K.kv_remap(a.table, a.kv_len, back, None, pool, h1, h2, b)
        K.kv_copy(cs, b)

    state = [pool.shares, pool.free_pages, a.table, a.kv_len, a.copies, a.meta, b.table, b.kv_len,
             b.copies, b.meta, h1, h2] + xs
    keep = [t.clone() for t in state]

    def reset():
        for t, k in zip(state, keep):
            t.copy_(k)

    lens.copy_(i32([40, 1, 96, 17, 32]))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        lens.copy_(i32(rng.integers(0, most * page + 1, B)))
        src.copy_(i32(np.sort(rng.integers(0, B, N))))
        back.copy_(i32(rng.integers(-1, N, B)))
        reset()
        call()
        want = [t.clone() for t in state]
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(state, want):
            assert torch.equal(t, w)
