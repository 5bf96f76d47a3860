"""include/plora_pages.h without a GPU: the library exports what the header declares, host
checks return the documented codes before anything is launched, the binding's refusals,
and the oracle's own pins."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import pages as OG
from paper_2608_05483_amd import pages as K
from paper_2608_05483_amd import paged as G
from paper_2608_05483_amd import plora as P
from test_paged_abi import FAKE, INV, OK, SMALL, UNS, cache, step

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "plora_pages.h")


def test_header_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(plora_[a-z_]+)\s*\(", text))
    assert names == set(K.EXPORTED)
    lib = ctypes.CDLL(P.LIB_PATH)
    for fn in names:
        assert hasattr(lib, fn), fn
    assert f"#define PLORA_CACHE_MAX_LAYERS {K.MAX_LAYERS}\n" in text


def pool(**kw):
    p = dict(n_pages=9, n_free=5, shares=FAKE, free_pages=FAKE, scratch=FAKE)
    p.update(kw)
    return K.plora_page_pool(**p)


def batch(**kw):
    b = dict(batch=3, max_pages=4, table=FAKE, kv_len=FAKE)
    b.update(kw)
    return K.plora_kv_batch(**b)


def new(**kw):
    return batch(**dict(dict(table=FAKE + 4096, kv_len=FAKE + 4096), **kw))


def remap_status(o=None, n=None, p=None, src=FAKE, keep=None, page=16, head=FAKE, nxt=FAKE + 64,
                 copies=FAKE, meta=FAKE, ws=FAKE, wb=None):
    o, n, p = o or batch(), n or new(), p or pool()
    wb = K.kv_remap_workspace_bytes(3, 3) if wb is None else wb
    return P.lib.plora_kv_remap(ctypes.byref(o), src, keep, page, ctypes.byref(p), head, nxt,
                                ctypes.byref(n), copies, meta, ws, wb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(o=batch(batch=-1)), INV), (dict(n=new(batch=-1)), INV),
    (dict(o=batch(max_pages=-1)), INV), (dict(n=new(max_pages=-1)), INV),
    (dict(p=pool(n_pages=-1)), INV), (dict(p=pool(n_free=-1)), INV),
    (dict(p=pool(shares=None)), INV), (dict(p=pool(free_pages=None)), INV),
    (dict(p=pool(scratch=None)), INV), (dict(src=None), INV), (dict(head=None), INV),
    (dict(nxt=None), INV), (dict(copies=None), INV), (dict(meta=None), INV), (dict(ws=None), INV),
    (dict(o=batch(table=None)), INV), (dict(o=batch(kv_len=None)), INV),
    (dict(n=new(table=None)), INV), (dict(n=new(kv_len=None)), INV),
    (dict(n=new(table=FAKE)), INV), (dict(n=new(kv_len=FAKE)), INV), (dict(nxt=FAKE), INV),
    (dict(src=FAKE + 4096), INV), (dict(keep=FAKE + 4096), INV),
    (dict(o=batch(batch=64, max_pages=1 << 25)), UNS),
    (dict(page=24), UNS), (dict(page=8), UNS), (dict(page=512), UNS),
    (dict(o=batch(batch=G.MAX_BATCH + 1)), UNS), (dict(n=new(batch=G.MAX_BATCH + 1)), UNS),
    (dict(o=batch(max_pages=(1 << 26) + 1)), UNS), (dict(n=new(max_pages=(1 << 26) + 1)), UNS),
    (dict(ws=FAKE + 8), UNS), (dict(p=pool(scratch=FAKE + 4)), UNS), (dict(wb=16), SMALL),
])
def test_remap_refusals(kw, want):
    assert remap_status(**kw) == want


def array(*cs):
    return (G.plora_kv_cache * len(cs))(*cs)


def copy_status(cs=None, layers=2, copies=FAKE, cap=3, n=FAKE):
    cs = array(cache(), cache()) if cs is None else cs
    return P.lib.plora_kv_copy(cs, layers, copies, cap, n, None)


def compact_status(cs=None, layers=2, s=None, path=FAKE, count=FAKE):
    cs = array(cache(), cache()) if cs is None else cs
    s = s or step()
    return P.lib.plora_kv_compact(cs, layers, ctypes.byref(s), path, count, None)


CACHES = [
    (dict(layers=-1), INV), (dict(layers=K.MAX_LAYERS + 1), UNS),
    (dict(cs=array(cache(k=None), cache())), INV), (dict(cs=array(cache(), cache(v=None))), INV),
    (dict(cs=array(cache(), cache(n_pages=7))), INV), (dict(cs=array(cache(), cache(dtype=1))), INV),
    (dict(cs=array(cache(), cache(head_stride=4096))), INV),
    (dict(cs=array(cache(), cache(kv_heads=1))), INV),
    (dict(cs=array(cache(), cache(token_stride=256))), INV),
    (dict(cs=array(cache(page_stride=-1), cache(page_stride=-1))), INV),
    (dict(cs=array(cache(n_pages=-1)), layers=1), INV),
    (dict(cs=array(cache(page_size=24)), layers=1), UNS),
    (dict(cs=array(cache(dtype=2)), layers=1), UNS),
    (dict(cs=array(cache(head_dim=514)), layers=1), UNS),
    (dict(cs=array(cache(kv_heads=1025)), layers=1), UNS),
    (dict(cs=array(cache(k=FAKE + 1)), layers=1), UNS),
]


@pytest.mark.parametrize("kw,want", CACHES + [
    (dict(copies=None), INV), (dict(n=None), INV), (dict(cap=-1), INV),
    (dict(cap=G.MAX_BATCH + 1), UNS), (dict(cap=0, copies=None, n=None), OK),
    (dict(layers=0), OK), (dict(cs=array(cache(kv_heads=0)), layers=1), OK),
])
def test_copy_refusals(kw, want):
    assert copy_status(**kw) == want


@pytest.mark.parametrize("kw,want", CACHES + [
    (dict(path=None), INV), (dict(count=None), INV), (dict(s=step(q_start=None)), INV),
    (dict(s=step(req=None)), INV), (dict(s=step(slot=None)), INV), (dict(s=step(batch=-1)), INV),
    (dict(s=step(T=-1)), INV), (dict(s=step(page_size=32)), INV),
    (dict(s=step(batch=G.MAX_BATCH + 1)), UNS), (dict(s=step(T=G.MAX_TOKENS + 1)), UNS),
    (dict(cs=array(cache(kv_heads=1024, head_dim=511)), layers=1,
          s=step(batch=G.MAX_BATCH)), UNS),
    (dict(s=step(batch=0), path=None), OK), (dict(s=step(T=0), path=None), OK),
    (dict(layers=0), OK),
])
def test_compact_refusals(kw, want):
    assert compact_status(**kw) == want


def test_sizes():
    assert K.kv_remap_workspace_bytes(-1, 3) == K.kv_remap_workspace_bytes(3, G.MAX_BATCH + 1) == 0
    assert K.kv_remap_workspace_bytes(0, 0) == 0
    assert 0 < K.kv_remap_workspace_bytes(1, 1) <= K.kv_remap_workspace_bytes(1000, 1)


def test_binding_refuses_what_pointers_cannot_tell():
    import torch
    i = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    for bad in ((i(4, dt=torch.int64), i(4)), (i(4), i(4, dt=torch.int64)), (i(8)[::2], i(4))):
        with pytest.raises(ValueError):
            K.PagePool(*bad)
    p = K.PagePool(i(9), i(5))
    r = K.Remap(2, 3, 16, 4, device="cpu")
    good = dict(table=i(2, 4), kv_len=i(2), src=i(3), keep=i(3), head=i(1), nxt=i(1))
    for kw in (dict(table=i(8)), dict(table=i(1, 4)), dict(table=i(2, 8)[:, ::2]),
               dict(table=i(2, 4, dt=torch.int64)), dict(kv_len=i(1)), dict(src=i(2)),
               dict(src=i(3, dt=torch.int64)), dict(keep=i(2)), dict(head=i(0)),
               dict(nxt=i(1, dt=torch.int64)), dict()):      # (the last: all on the host)
        a = dict(good, **kw)
        with pytest.raises(ValueError):
            K.kv_remap(a["table"], a["kv_len"], a["src"], a["keep"], p, a["head"], a["nxt"], r)
    with pytest.raises(ValueError):
        K.Remap(2, 3, 16, 4, device="cpu", table=i(3, 5))
    c = lambda *s, **k: G.KVCache(z(*s, **k), z(*s, **k))
    for x in (c(3, 2, 16, 32), c(3, 2, 32, 64), c(4, 2, 16, 64), c(3, 2, 16, 64, dt=torch.float16),
              G.KVCache(z(3, 16, 2, 64).transpose(1, 2), z(3, 16, 2, 64).transpose(1, 2))):
        with pytest.raises(ValueError):
            K.Caches([c(3, 2, 16, 64), x])
    with pytest.raises(ValueError):
        K.Caches([c(1, 1, 16, 2)] * (K.MAX_LAYERS + 1))
    cs = K.Caches([c(3, 2, 16, 64)] * 2)
    with pytest.raises(ValueError):
        K.kv_copy(cs, K.Remap(2, 3, 32, 4, device="cpu"))
    s = G.Step(2, 5, 16, 3, device="cpu")
    for path, count in ((i(4), i(2)), (i(5), i(1)), (i(5, dt=torch.int64), i(2)), (i(5), i(2))):
        with pytest.raises(ValueError):
            K.kv_compact(cs, s, path, count)
    K.kv_copy(K.Caches([]), r), K.kv_compact(K.Caches([]), s, i(5), i(2))    # nothing to do


# ---- the oracle's pins ------------------------------------------------------------------


def test_oracle_remap():
    """One request of 20 keys on pages 7, 3 continued by three; then two of them end."""
    table, shares, free = np.array([[7, 3, -1]]), [0] * 8, [9, 9, 0, 1, 2]
    new = np.full((3, 3), -1)
    got = OG.remap(table, [20], [0, 0, 0], None, 16, shares, free, 2, new)
    assert new.tolist() == [[7, 0, -1], [7, 1, -1], [7, 3, -1]]
    assert shares == [0, 0, 0, 0, 0, 0, 0, 2] and got["next"] == 4
    assert got["copies"].tolist() == [[3, 0, 4], [3, 1, 4], [-1] * 3]
    assert got["meta"] == [0, 2, 0, 0, 0, 0, 0, 0] and got["kv_len"] == [20] * 3
    last = np.full((1, 3), -1)
    got = OG.remap(new, [20] * 3, [1], [17], 16, shares, free, 4, last)
    assert last.tolist() == [[7, 1, -1]] and shares == [0] * 8
    assert free == [9, 9, 0, 3, 2] and got["next"] == 2 and got["meta"][:4] == [2, 0, 0, 0]
    # cut inside a page that another holds whole: a page of its own
    got = OG.remap(np.array([[4, 5]]), [32], [0, 0], [32, 20], 16, shares, free, 4,
                   np.full((2, 2), -1))
    assert got["copies"].tolist() == [[5, 2, 4], [-1] * 3] and shares[4] == 1 and shares[5] == 0
    # nothing in the list: the request ends at its last whole page
    got = OG.remap(np.array([[4, 5]]), [32], [0, 0], [32, 20], 16, [0] * 8, free, 5,
                   np.full((2, 2), -1))
    assert got["kv_len"] == [32, 16] and got["meta"][:4] == [0, 0, 1, 0]


def test_oracle_moves():
    x = np.arange(3 * 2 * 4 * 1.0).reshape(3, 2, 4, 1)
    y = x.copy()
    OG.copy(y, [(0, 2, 3), (1, 0, 9), (5, 1, 2)], 2)
    assert (y[2, :, :3] == x[0, :, :3]).all() and (y[2, :, 3] == x[2, :, 3]).all()
    assert (y[0] == x[1]).all() and (y[1] == x[1]).all()
    y = x.copy()
    OG.compact(y, [0, 4], [0] * 4, [2, 3, 8, 9], [0, 2, 3, 1], [3])
    assert (y[0, :, 3] == x[2, :, 0]).all() and (y[2, :, 0] == x[2, :, 1]).all()
    assert (y[0, :, 2] == x[0, :, 2]).all() and (y[2, :, 1] == x[2, :, 1]).all()
