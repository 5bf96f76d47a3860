"""include/plora_paged.h without a GPU: the library exports what the header
declares, host checks return the documented codes before anything is launched,
sizes and bounds, the rotation's frequencies, and the oracle's own pins."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from oracle import paged as OP
from paper_2608_05483_amd import paged as G
from paper_2608_05483_amd import plora as P

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "plora_paged.h")
FAKE = 0x10000  # an aligned non-null address; never dereferenced by these checks
OK, INV, UNS, SMALL = (P.PLORA_OK, P.PLORA_ERR_INVALID_ARG, P.PLORA_ERR_UNSUPPORTED,
                       P.PLORA_ERR_WORKSPACE_TOO_SMALL)


def test_header_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(plora_[a-z_]+)\s*\(", text))
    assert names == set(G.EXPORTED)
    lib = ctypes.CDLL(P.LIB_PATH)
    for fn in names:
        assert hasattr(lib, fn), fn
    consts = dict(re.findall(r"#define (PLORA_\w+) (\d+)\n", text))
    assert int(consts["PLORA_PAGED_MAX_BATCH"]) == G.MAX_BATCH
    assert int(consts["PLORA_PAGED_MAX_TOKENS"]) == G.MAX_TOKENS
    assert int(consts["PLORA_PAGE_MIN"]) == G.PAGE_MIN
    assert int(consts["PLORA_PAGE_MAX"]) == G.PAGE_MAX
    assert int(consts["PLORA_ATTN_SHARE_ROWS"]) == G.SHARE_ROWS


def step(**kw):
    s = dict(batch=4, T=8, page_size=16, max_pages=10, table=FAKE, q_start=FAKE, kv_len=FAKE,
             pos=FAKE, req=FAKE, slot=FAKE, meta=FAKE)
    s.update(kw)
    return G.plora_kv_step(**s)


def plan_status(s=None, past=FAKE, new=FAKE, free=FAKE, n_free=4, head=FAKE, nxt=FAKE):
    s = s or step()
    return P.lib.plora_kv_plan(past, new, free, n_free, head, nxt, ctypes.byref(s), None)


@pytest.mark.parametrize("kw,want", [
    (dict(s=step(batch=-1)), INV), (dict(s=step(T=-1)), INV), (dict(s=step(max_pages=-1)), INV),
    (dict(n_free=-1), INV), (dict(head=None), INV), (dict(nxt=None), INV), (dict(past=None), INV),
    (dict(new=None), INV), (dict(free=None), INV), (dict(s=step(table=None)), INV),
    (dict(s=step(q_start=None)), INV), (dict(s=step(kv_len=None)), INV),
    (dict(s=step(pos=None)), INV), (dict(s=step(req=None)), INV), (dict(s=step(slot=None)), INV),
    (dict(s=step(meta=None)), INV), (dict(s=step(page_size=24)), UNS),
    (dict(s=step(page_size=8)), UNS), (dict(s=step(page_size=512)), UNS),
    (dict(s=step(batch=G.MAX_BATCH + 1)), UNS), (dict(s=step(T=G.MAX_TOKENS + 1)), UNS),
    (dict(s=step(max_pages=(1 << 26) + 1)), UNS),
])
def test_kv_plan_refusals(kw, want):
    assert plan_status(**kw) == want


def rope_status(x=FAKE, xt=256, xh=128, pos=FAKE, turns=FAKE, T=4, H=2, D=128, rot=64, layout=0,
                scale=1.0, inverse=0, dt=0, out=FAKE, ot=256, oh=128):
    return P.lib.plora_rope(x, xt, xh, pos, turns, T, H, D, rot, layout, scale, inverse, dt, out,
                            ot, oh, None)


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), INV), (dict(H=-1), INV), (dict(D=-2), INV), (dict(rot=130), INV),
    (dict(rot=-2), INV), (dict(x=None), INV), (dict(out=None), INV), (dict(pos=None), INV),
    (dict(turns=None), INV), (dict(xt=-1), INV), (dict(oh=-1), INV),
    (dict(scale=math.inf), INV), (dict(scale=math.nan), INV), (dict(rot=63), UNS),
    (dict(D=127, rot=2), UNS), (dict(D=514), UNS), (dict(layout=2), UNS), (dict(dt=2), UNS),
    (dict(x=FAKE + 1), UNS), (dict(T=G.MAX_TOKENS + 1), UNS), (dict(T=0, x=None), OK),
    (dict(H=0, x=None), OK), (dict(D=0, rot=0, x=None), OK),
])
def test_rope_refusals(kw, want):
    assert rope_status(**kw) == want


def cache(**kw):
    c = dict(n_pages=6, page_size=16, kv_heads=2, head_dim=128, dtype=0, reserved=0, k=FAKE,
             v=FAKE, page_stride=2 * 16 * 128, head_stride=16 * 128, token_stride=128)
    c.update(kw)
    return G.plora_kv_cache(**c)


def append_status(c=None, q=FAKE, k=FAKE, v=FAKE, pos=FAKE, slot=FAKE, turns=FAKE, T=4, H=2,
                  rot=64, layout=0, scale=1.0, out=FAKE, qt=256, kt=256, vt=256, ot=256):
    c = c or cache()
    return P.lib.plora_rope_append(q, qt, 128, k, kt, 128, v, vt, 128, pos, slot, turns, T, H,
                                   rot, layout, scale, ctypes.byref(c), out, ot, 128, None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(pos=None), INV),
    (dict(slot=None), INV), (dict(turns=None), INV), (dict(out=None), INV), (dict(qt=-8), INV),
    (dict(kt=-8), INV), (dict(vt=-8), INV), (dict(ot=-8), INV), (dict(rot=200), INV),
    (dict(c=cache(k=None)), INV), (dict(c=cache(n_pages=-1)), INV),
    (dict(c=cache(kv_heads=-1)), INV), (dict(c=cache(page_stride=-1)), INV),
    (dict(c=cache(page_size=17)), UNS), (dict(c=cache(dtype=5)), UNS),
    (dict(c=cache(head_dim=1024)), UNS), (dict(rot=33), UNS), (dict(k=FAKE + 1), UNS),
    (dict(T=0, q=None), OK),
])
def test_rope_append_refusals(kw, want):
    assert append_status(**kw) == want


def shape(**kw):
    s = dict(batch=4, T=8, heads=8, kv_heads=2, head_dim=128, max_q=4, shared=0, reserved=0)
    s.update(kw)
    return G.plora_attn_shape(**s)


def seg(T=4, n=3, **kw):
    s = dict(T=T, cap=min(T, n), tile_cap=P.plora_tile_capacity(T, n), reserved=0, perm=FAKE,
             seg_ptr=FAKE, seg_id=FAKE, meta=FAKE, tiles=FAKE)
    s.update(kw)
    return P.plora_segments(**s)


def attn_plan_status(s=None, sh=None, g=None, prefix=FAKE, n=0, plan=FAKE, nbytes=None):
    s, sh = s or step(), sh or shape()
    nbytes = G.attn_plan_bytes(sh) if nbytes is None else nbytes
    return P.lib.plora_attn_plan(ctypes.byref(s), ctypes.byref(sh),
                                 ctypes.byref(g) if g is not None else None, prefix, n, plan,
                                 nbytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(sh=shape(batch=5)), INV), (dict(sh=shape(T=9)), INV), (dict(sh=shape(heads=-8)), INV),
    (dict(sh=shape(max_q=-1)), INV), (dict(s=step(req=None)), INV),
    (dict(s=step(kv_len=None)), INV), (dict(s=step(q_start=None)), INV), (dict(plan=None), INV),
    (dict(g=seg(), n=3), INV),                                   # groups without shape.shared
    (dict(sh=shape(shared=1), g=seg(), n=3, prefix=None), INV),
    (dict(sh=shape(shared=1), g=seg(perm=None), n=3), INV),
    (dict(sh=shape(shared=1), g=seg(T=5), n=3), INV),
    (dict(sh=shape(shared=1), g=seg(cap=2), n=3), INV), (dict(n=-1), INV),
    (dict(sh=shape(heads=9)), UNS), (dict(sh=shape(head_dim=96)), UNS),
    (dict(s=step(page_size=20)), UNS), (dict(plan=FAKE + 4), UNS), (dict(nbytes=16), SMALL),
    (dict(s=step(batch=0), sh=shape(batch=0), plan=None), OK),
    (dict(s=step(T=0), sh=shape(T=0), plan=None), OK), (dict(sh=shape(heads=0), plan=None), OK),
])
def test_attn_plan_refusals(kw, want):
    assert attn_plan_status(**kw) == want


def attn_status(s=None, sh=None, c=None, q=FAKE, out=FAKE, plan=FAKE, ws=FAKE, scale=0.1,
                qt=1024, qh=128, ot=1024, oh=128, pb=None, wb=None):
    s, sh, c = s or step(), sh or shape(), c or cache()
    pb = G.attn_plan_bytes(sh) if pb is None else pb
    wb = G.attn_paged_workspace_bytes(sh) if wb is None else wb
    return P.lib.plora_attn_paged(q, qt, qh, ctypes.byref(c), ctypes.byref(s), ctypes.byref(sh),
                                  scale, plan, pb, out, ot, oh, ws, wb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INV), (dict(out=None), INV), (dict(plan=None), INV), (dict(ws=None), INV),
    (dict(scale=math.nan), INV), (dict(scale=math.inf), INV), (dict(qt=-8), INV),
    (dict(oh=-8), INV), (dict(c=cache(kv_heads=4)), INV), (dict(c=cache(head_dim=64)), INV),
    (dict(c=cache(page_size=32)), INV), (dict(c=cache(k=None)), INV),
    (dict(c=cache(token_stride=120)), INV), (dict(s=step(batch=3)), INV),
    (dict(s=step(table=None)), INV), (dict(s=step(pos=None)), INV), (dict(s=step(req=None)), INV),
    (dict(qt=1020), UNS), (dict(qh=132), UNS), (dict(ot=1028), UNS),
    (dict(c=cache(token_stride=132)), UNS), (dict(c=cache(dtype=3)), UNS),
    (dict(c=cache(page_stride=4100)), UNS), (dict(c=cache(token_stride=1 << 30)), UNS),
    (dict(q=FAKE + 2), UNS), (dict(out=FAKE + 8), UNS), (dict(ws=FAKE + 8), UNS),
    (dict(c=cache(v=FAKE + 8)), UNS), (dict(pb=64), SMALL), (dict(wb=64), SMALL),
    (dict(s=step(T=0), sh=shape(T=0), q=None), OK), (dict(sh=shape(heads=0), q=None), OK),
])
def test_attn_paged_refusals(kw, want):
    assert attn_status(**kw) == want


def test_a_launch_of_too_many_threads_is_refused():
    big = dict(batch=1, T=1 << 20)
    assert attn_status(s=step(**big), sh=shape(heads=65536, kv_heads=1024, max_q=1 << 20, **big),
                       c=cache(kv_heads=1024)) == UNS


def test_sizes():
    assert G.attn_plan_bytes(shape(batch=0)) == 0 and G.attn_plan_bytes(shape(T=0)) == 0
    assert G.attn_plan_bytes(shape(heads=7)) == 0
    assert G.attn_paged_workspace_bytes(shape(head_dim=96)) == 0
    # a decode batch takes no tile items, a shared one does
    a, b = shape(max_q=1), shape(max_q=1, shared=1)
    assert 0 < G.attn_plan_bytes(a) < G.attn_plan_bytes(b)
    assert 0 < G.attn_paged_workspace_bytes(a) < G.attn_paged_workspace_bytes(b)


def test_binding_refuses_what_pointers_cannot_tell():
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    c = G.KVCache(z(3, 2, 16, 64), z(3, 2, 16, 64))
    for k, v in [(z(3, 2, 16), z(3, 2, 16)), (z(3, 2, 16, 64), z(3, 2, 16, 32)),
                 (z(3, 2, 64, 16).transpose(2, 3), z(3, 2, 64, 16).transpose(2, 3)),
                 (z(3, 2, 16, 64), z(3, 16, 2, 64).transpose(1, 2))]:
        with pytest.raises(ValueError):
            G.KVCache(k, v)
    with pytest.raises(TypeError):
        G.KVCache(z(3, 2, 16, 64, dt=torch.float32), z(3, 2, 16, 64, dt=torch.float32))
    i = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    q, k = z(5, 4, 64), z(5, 2, 64)
    bad = [dict(k=z(5, 3, 64)), dict(q=z(5, 4, 32)), dict(q_out=z(5, 3, 64)), dict(pos=i(4)),
           dict(pos=i(5, torch.int64)), dict(slot=i(5)), dict(turns=i(32)),
           dict(q=z(5, 64, 4).transpose(1, 2))]
    for kw in bad:
        a = dict(q=q, k=k, v=k, pos=i(5), slot=i(5, torch.int64), turns=i(32, torch.int64),
                 q_out=q)
        a.update(kw)
        with pytest.raises(ValueError):
            G.rope_append(a["q"], a["k"], a["v"], a["pos"], a["slot"], a["turns"], c, a["q_out"])
    with pytest.raises(TypeError):
        G.rope_append(q.half(), k, k, i(5), i(5, torch.int64), i(32, torch.int64), c, q)
    with pytest.raises(ValueError):
        G.Step(3, 4, 16, 5, device="cpu", table=i(14))


# ---- the rotation's frequencies -------------------------------------------------------


def turns(**kw):
    t = G.rope_turns(device="cpu", **kw)
    return [int(x) for x in t.numpy().view(np.uint64)]


def radians(t):
    return np.array([x / 2.0 ** 64 * 2 * math.pi for x in t])


def test_turns():
    assert turns(rot=0) == []
    plain = radians(turns(rot=64))
    want = [10000.0 ** (-2 * i / 64) for i in range(32)]
    assert np.allclose(plain, want, rtol=1e-14)
    assert np.allclose(radians(turns(rot=64, scaling="linear", factor=4.0)), plain / 4, rtol=1e-14)
    base = radians(turns(rot=64, scaling="base", factor=8.0))
    assert math.isclose(base[0], plain[0], rel_tol=1e-14)
    assert math.isclose(base[-1], plain[-1] / 8, rel_tol=1e-12)
    band = radians(turns(rot=64, scaling="bands", factor=8.0, original=4096))
    made = 4096 * plain / (2 * math.pi)
    assert np.allclose(band[made >= 32], plain[made >= 32], rtol=1e-14)
    assert np.allclose(band[made <= 1], plain[made <= 1] / 8, rtol=1e-14)
    mid = (made > 1) & (made < 32)
    assert mid.any() and (band[mid] < plain[mid]).all() and (band[mid] > plain[mid] / 8).all()
    for kw in (dict(rot=3), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, factor=0.0),
               dict(rot=8, scaling="bands"), dict(rot=8, scaling="other"),
               dict(rot=8, scaling="bands", original=9, low=3.0, high=2.0)):
        with pytest.raises(ValueError):
            turns(**kw)


# ---- the oracle's pins ------------------------------------------------------------------


def test_oracle_rotation():
    x = np.arange(24.0).reshape(2, 2, 6)
    # a quarter turn a position, and none
    t = [2 ** 62, 0]
    half = OP.rotate(x, [1, 3], t, "half")
    assert np.allclose(half[0, :, [0, 2]], np.stack([-x[0, :, 2], x[0, :, 0]]))
    assert np.allclose(half[1, :, [0, 2]], np.stack([x[1, :, 2], -x[1, :, 0]]))
    assert np.array_equal(half[..., [1, 3, 4, 5]], x[..., [1, 3, 4, 5]])
    pair = OP.rotate(x, [1, 3], t, "interleaved", scale=2.0)
    assert np.allclose(pair[0, :, 0], -2 * x[0, :, 1]) and np.allclose(pair[0, :, 1], 2 * x[0, :, 0])
    # the inverse undoes it, and lengths are kept
    t = [123456789 << 30, 987654321 << 20, 5]
    y = OP.rotate(x, [100, 10 ** 9], t, "half")
    assert np.allclose(OP.rotate(y, [100, 10 ** 9], t, "half", inverse=True), x)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))


def test_oracle_plan_by_hand():
    table = np.full((3, 4), -1)
    table[0, 0] = 9
    r = OP.kv_plan([3, 0, 16], [2, 17, 0], [50, 51, 52], 0, table, 16, 20)
    assert r["q_start"] == [0, 2, 19, 19] and r["kv_len"] == [5, 17, 16]
    assert r["pos"][:4] == [3, 4, 0, 1] and r["req"] == [0, 0] + [1] * 17 + [-1]
    assert r["slot"][:3] == [9 * 16 + 3, 9 * 16 + 4, 50 * 16] and r["slot"][18:] == [51 * 16, -1]
    assert r["next"] == 2 and r["meta"][:3] == [19, 2, 0] and list(table[1, :2]) == [50, 51]


def test_oracle_attention_equals_the_decode_oracle():
    """On a cache that is one page a request, one token each: the contiguous
    decode attention's oracle, which is pinned by itself."""
    import oracle
    from oracle import attention as OA
    rng = np.random.default_rng(0)
    B, H, L, D = 3, 2, 16, 8
    bits = lambda *s: oracle.f32_to_bf16(rng.normal(size=s).astype(np.float32))
    q, k, v = bits(B, H, D), bits(B, H, L, D), bits(B, H, L, D)
    lens = np.array([16, 1, 7])
    want = OA.attention(q, k, v, lens, 0.4)
    f = lambda a: oracle.bf16_to_f32(a).astype(np.float64)
    got, size = OP.attention(f(q), f(k), f(v), np.arange(B)[:, None], None, None,
                             np.arange(B), lens - 1, L, 0.4)
    assert np.allclose(got, want) and (size >= np.abs(got) - 1e-12).all()


def test_step_is_laid_out_for_a_shape_that_cannot_overflow():
    """The bounds of items and partial rows hold for any lengths: a model of the
    cuts in whole numbers, over random batches."""
    rng = np.random.default_rng(5)
    few, tile, few_target, tile_target = 16, 128, FEW_TARGET, TILE_TARGET
    for _ in range(300):
        B = int(rng.integers(1, 60))
        r, KH = int(rng.choice([1, 3, 8, 16, 20])), int(rng.choice([1, 2, 8, 32]))
        new = rng.integers(0, int(rng.choice([2, 9, 400])) + 1, B)
        kv = new + rng.integers(0, int(rng.choice([1, 500, 20000])) + 1, B)
        T, max_q = int(new.sum()), int(new.max())
        shared = bool(rng.integers(0, 2))
        sets = []                                       # (rows, keys, partials always)
        u = np.zeros(B, int)
        if shared:
            group = rng.integers(0, 4, B)
            for g in range(4):
                mem = [b for b in range(B) if group[b] == g and new[b] and new[b] * r <= 128]
                length = min([int(kv[b] - new[b]) for b in mem], default=0) // 16 * 16
                if len(mem) >= 2 and length:
                    u[mem] = length
                    sets.append((int(new[mem].sum()) * r, length, True))
        sets += [(int(new[b]) * r, int(kv[b] - u[b]), u[b] > 0) for b in range(B) if new[b]]
        tiles = lambda n: 1 if n <= few else -(-n // tile)
        work = [sum(tiles(n) * k for n, k, _ in sets if (n <= few) == f) for f in (True, False)]
        per = [max(256, -(-w // -(-t // KH))) for w, t in zip(work, (few_target, tile_target))]
        items, rows = [0, 0], 0
        for n, k, always in sets:
            i = 0 if n <= few else 1
            pieces = -(-k // per[i])
            items[i] += tiles(n) * pieces
            rows += n * pieces if always or pieces > 1 else 0
        more = [-(-few_target // KH), -(-tile_target // KH)]
        sharing = min(T * r, B * 128) if shared else 0
        has_tiles = shared or max_q * r > few
        assert items[0] <= B + (B // 2 if shared else 0) + more[0]
        assert items[1] <= ((T * r // tile + min(B, T * r // 17) + sharing // tile
                             + (B // 2 if shared else 0) + more[1]) if has_tiles else 0)
        least = few if shared else min(few, max_q * r)
        assert rows <= 2 * sharing + 2 * (least * more[0] + (tile * more[1] if has_tiles else 0))


def _constant(name):
    text = open(os.path.join(os.path.dirname(P.__file__), "csrc", "paged", "attn_plan.h")).read()
    return int(re.search(rf"constexpr int {name} = (\d+);", text).group(1))


FEW_TARGET, TILE_TARGET = _constant("kFewTarget"), _constant("kTileTarget")


@pytest.mark.parametrize("page", [16, 128, 256])
def test_longest_token_stride(page):
    """A cache's keys may lie up to 2^25 elements apart, whatever the page size."""
    for stride, want in ((1 << 25, UNS), ((1 << 25) - 8, SMALL)):
        assert attn_status(c=cache(page_size=page, token_stride=stride), s=step(page_size=page),
                           wb=64) == want


def test_binding_refuses_host_tensors():
    """No call hands the address of a host tensor to a kernel."""
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    i = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    c = G.KVCache(z(3, 2, 16, 64), z(3, 2, 16, 64))
    s = G.Step(2, 5, 16, 4, device="cpu")
    p = G.AttnPlan(s, 4, 2, 64, max_q=3, device="cpu")
    q, k = z(5, 4, 64), z(5, 2, 64)
    turns = i(32, torch.int64)
    for call in (lambda: G.kv_plan(i(2), i(2), i(3), i(1), i(1), s),
                 lambda: G.rope(q, i(5), turns, q),
                 lambda: G.rope_append(q, k, k, i(5), i(5, torch.int64), turns, c, q),
                 lambda: G.attn_plan(s, p), lambda: G.attn_paged(q, c, s, p, 0.1, q.clone())):
        with pytest.raises(ValueError, match="GPU tensors"):
            call()


def test_the_plan_s_count_is_where_the_header_says():
    text = open(HEADER).read()
    assert int(re.search(r"#define PLORA_ATTN_PLAN_LEFT_OUT (\d+)", text).group(1)) == \
        G.PLAN_LEFT_OUT


def test_oracle_keeps_requests_of_no_tokens():
    r = OP.kv_plan([16, 16, 16], [0, 30, 0], [1, 2, 3], 0, np.zeros((3, 4), int), 16, 20)
    assert r["meta"][:3] == [20, 0, 1] and r["kv_len"] == [16, 16, 16]


def test_a_failed_launch_names_its_error():
    """Where there is no GPU, a launch fails with the runtime's "no device"."""
    import torch
    if torch.cuda.device_count():
        pytest.skip("launches succeed here")
    assert plan_status() == P.PLORA_ERR_HIP
    assert P.lib.plora_paged_last_hip_error() == 100
    assert attn_plan_status() == rope_status() == append_status() == attn_status() == \
        P.PLORA_ERR_HIP
    with pytest.raises(P.PloraError, match="hipError_t 100"):
        G._ok("plora_rope", rope_status())


def test_a_table_of_other_rows_is_refused():
    """Rows of another length than max_pages would be read as each other's pages; more
    rows than requests, or a flat table, are fine."""
    import torch
    t = lambda *s: torch.zeros(s, dtype=torch.int32)
    for bad in (t(3, 6), t(4, 4), t(3, 4), t(2, 5), t(3, 10)[:, :5], t(3, 5, 2)):
        with pytest.raises(ValueError):
            G.Step(3, 4, 16, 5, device="cpu", table=bad)
    for good in (t(3, 5), t(9, 5), t(15)):
        assert G.Step(3, 4, 16, 5, device="cpu", table=good).table is good
