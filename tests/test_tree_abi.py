"""include/plora_tree.h without a GPU: the library exports what the header declares, host
checks return the documented codes before anything is launched, the binding's refusals,
and the oracle's own pins."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from oracle import tree as OT
from paper_2608_05483_amd import paged as G
from paper_2608_05483_amd import plora as P
from paper_2608_05483_amd import tree as R
from test_paged_abi import FAKE, INV, OK, SMALL, UNS, cache, shape, step

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "plora_tree.h")


def test_header_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(plora_[a-z_]+)\s*\(", text))
    assert names == set(R.EXPORTED)
    lib = ctypes.CDLL(P.LIB_PATH)
    for fn in names:
        assert hasattr(lib, fn), fn
    assert f"#define PLORA_TREE_MAX_NODES {R.MAX_NODES}\n" in text
    assert R.MAX_NODES == OT.MAX_NODES


def tree(**kw):
    t = dict(batch=4, T=8, pos=FAKE, span=FAKE, info=FAKE)
    t.update(kw)
    return R.plora_tree(**t)


def plan_status(s=None, t=None, parent=FAKE):
    s, t = s or step(), t or tree()
    return P.lib.plora_tree_plan(parent, ctypes.byref(s), ctypes.byref(t), None)


@pytest.mark.parametrize("kw,want", [
    (dict(s=step(batch=-1), t=tree(batch=-1)), INV), (dict(s=step(T=-1), t=tree(T=-1)), INV),
    (dict(t=tree(batch=3)), INV), (dict(t=tree(T=9)), INV), (dict(parent=None), INV),
    (dict(t=tree(pos=None)), INV), (dict(t=tree(span=None)), INV), (dict(t=tree(info=None)), INV),
    (dict(s=step(q_start=None)), INV), (dict(s=step(kv_len=None)), INV),
    (dict(s=step(req=None)), INV),
    (dict(s=step(batch=G.MAX_BATCH + 1), t=tree(batch=G.MAX_BATCH + 1)), UNS),
    (dict(s=step(T=G.MAX_TOKENS + 1), t=tree(T=G.MAX_TOKENS + 1)), UNS),
    (dict(t=tree(span=FAKE + 4)), UNS), (dict(t=tree(info=FAKE + 4)), UNS),
    (dict(s=step(batch=0, T=0), t=tree(batch=0, T=0), parent=None), OK),
])
def test_tree_plan_refusals(kw, want):
    assert plan_status(**kw) == want


def attn_status(s=None, sh=None, c=None, t=None, q=FAKE, out=FAKE, plan=FAKE, ws=FAKE, scale=0.1,
                qt=1024, qh=128, ot=1024, oh=128, pb=None, wb=None, no_tree=False):
    s, sh, c, t = s or step(), sh or shape(), c or cache(), t or tree()
    pb = G.attn_plan_bytes(sh) if pb is None else pb
    wb = G.attn_paged_workspace_bytes(sh) if wb is None else wb
    return P.lib.plora_attn_tree(q, qt, qh, ctypes.byref(c), ctypes.byref(s), ctypes.byref(sh),
                                 None if no_tree else ctypes.byref(t), scale, plan, pb, out, ot,
                                 oh, ws, wb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(no_tree=True), INV), (dict(t=tree(batch=3)), INV), (dict(t=tree(T=7)), INV),
    (dict(t=tree(span=None)), INV), (dict(t=tree(info=None)), INV),
    (dict(t=tree(span=FAKE + 4)), UNS), (dict(t=tree(info=FAKE + 4)), UNS),
    (dict(q=None), INV), (dict(out=None), INV), (dict(plan=None), INV), (dict(ws=None), INV),
    (dict(scale=math.nan), INV), (dict(qt=-8), INV), (dict(c=cache(kv_heads=4)), INV),
    (dict(s=step(pos=None)), INV), (dict(s=step(table=None)), INV),
    (dict(c=cache(token_stride=120)), INV), (dict(qt=1020), UNS), (dict(q=FAKE + 2), UNS),
    (dict(c=cache(dtype=3)), UNS), (dict(sh=shape(head_dim=96), c=cache(head_dim=96)), UNS),
    (dict(pb=64), SMALL), (dict(wb=64), SMALL),
    (dict(s=step(T=0), sh=shape(T=0), t=tree(T=0), q=None), OK),
    (dict(sh=shape(heads=0), q=None), OK),
])
def test_attn_tree_refusals(kw, want):
    assert attn_status(**kw) == want


def accept_status(s=None, parent=FAKE, drafted=FAKE, target=FAKE, nb=4, given=FAKE, path=FAKE,
                  count=FAKE, token=FAKE, kv=FAKE + 4096):
    s = s or step()
    return P.lib.plora_tree_accept(parent, drafted, target, nb, given, ctypes.byref(s), path, count,
                                   token, kv, None)


@pytest.mark.parametrize("kw,want", [
    (dict(parent=None), INV), (dict(drafted=None), INV), (dict(target=None), INV),
    (dict(path=None), INV), (dict(count=None), INV), (dict(token=None), INV), (dict(kv=None), INV),
    (dict(s=step(q_start=None)), INV), (dict(s=step(kv_len=None)), INV),
    (dict(s=step(req=None)), INV), (dict(s=step(batch=-1)), INV), (dict(s=step(T=-1)), INV),
    (dict(kv=FAKE), INV), (dict(nb=2), UNS), (dict(nb=0), UNS), (dict(nb=8, drafted=FAKE + 4), UNS),
    (dict(nb=8, target=FAKE + 4), UNS), (dict(nb=8, token=FAKE + 4), UNS),
    (dict(s=step(batch=G.MAX_BATCH + 1)), UNS), (dict(s=step(T=G.MAX_TOKENS + 1)), UNS),
    (dict(s=step(batch=0, T=0), parent=None), OK),
])
def test_accept_refusals(kw, want):
    assert accept_status(**kw) == want


def test_binding_refuses_what_pointers_cannot_tell():
    import torch
    i = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    s = G.Step(2, 5, 16, 3, device="cpu")
    t = R.Tree(s, device="cpu")
    for parent in (i(4), i(5, torch.int64), i(10)[::2]):
        with pytest.raises(ValueError):
            R.tree_plan(parent, s, t)
    with pytest.raises(TypeError):
        R.Accepted(s, dtype=torch.int16, device="cpu")
    a = R.Accepted(s, device="cpu")
    good = dict(parent=i(5), drafted=i(5), target=i(5), given=i(2))
    for kw in (dict(parent=i(4)), dict(drafted=i(5, torch.int64)), dict(target=i(4)),
               dict(target=i(10)[::2]), dict(given=i(1)), dict(given=i(2, torch.int64))):
        x = dict(good, **kw)
        with pytest.raises(ValueError):
            R.tree_accept(x["parent"], x["drafted"], x["target"], s, a, x["given"])
    other = G.Step(2, 6, 16, 3, device="cpu")
    with pytest.raises(ValueError):
        R.tree_accept(i(6), i(6), i(6), other, a)
    with pytest.raises(ValueError):              # all on the host
        R.tree_plan(i(5), s, t)


def test_calls_are_made_with_the_tensors_gpu_current(monkeypatch):
    import torch
    now, seen = [0], []

    class Device:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            self.was, now[0] = now[0], self.d

        def __exit__(self, *a):
            now[0] = self.was

    monkeypatch.setattr(R, "_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for dev in (0, 3):
        R._launch("call", lambda *a: seen.append((now[0], a)) or OK, dev, 1, 2)
        with pytest.raises(P.PloraError):
            R._launch("call", lambda: INV, dev)
        assert now == [0]
    assert seen == [(0, (1, 2)), (3, (1, 2))]


# ---- the oracle's pins ------------------------------------------------------------------


def test_oracle_paths_and_numbers():
    #        0
    #      1   2      7 (a root of its own)
    #     3 4  5
    #          6
    par = [-1, 0, 0, 1, 1, 2, 5, -1, 8, -3, 9, 4]    # 8: its own parent, 9: out of range, 10: cut
    way = OT.paths(par)
    assert way[6] == [0, 2, 5, 6] and way[4] == [0, 1, 4] and way[7] == [7]
    assert way[11] == [0, 1, 4, 11] and way[8] is way[9] is way[10] is None
    got = OT.tree_plan(par, [0, 12], [100 + 12], [0] * 12, 12)
    assert got["pos"] == [100, 101, 101, 102, 102, 102, 103, 100, 0, 0, 0, 103]
    assert got["span"][:8] == [(0, 7), (1, 4), (5, 7), (2, 2), (3, 4), (6, 7), (7, 7), (8, 8)]
    assert got["span"][8:] == [(-1, -2)] * 3 + [(4, 4)] and got["info"] == [(1, 3)]
    first, last = np.array(got["span"]).T
    for i in range(12):
        for j in range(12):
            seen = way[i] is not None and j in way[i]
            assert seen == bool(first[j] <= first[i] <= last[j] and way[i] is not None)
    chain = OT.tree_plan([-1, 0, 1], [0, 3], [8], [0] * 3, 3)
    assert chain == dict(pos=[5, 6, 7], span=[(0, 2), (1, 2), (2, 2)], info=[(0, 0)])


def test_oracle_attention_of_a_chain_is_causal():
    from oracle import paged as OP
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(5, 2, 8)), rng.normal(size=(3, 1, 4, 8)), rng.normal(size=(3, 1, 4, 8))
    table = np.array([[2, 0, 1]])
    args = (q, k, v, table, [0, 5], [11], np.zeros(5, int))
    want = OP.attention(*args, np.arange(6, 11), 4, 0.3)
    got = OT.attention(*args, np.arange(5) - 1, 4, 0.3)
    assert np.allclose(got[0], want[0], atol=1e-14) and np.allclose(got[1], want[1], atol=1e-14)
    # roots see the cached keys and themselves: as if each were the only new token
    alone = OT.attention(*args, np.full(5, -1), 4, 0.3)
    flat = lambda x, t: x[table[0][t // 4], 0, t % 4]
    idx = np.r_[0:6, 9]
    s = 0.3 * q[3, 1] @ flat(k, idx).T
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(alone[0][3, 1], w @ flat(v, idx), atol=1e-13)


def test_oracle_accept():
    par = [-1, 0, 0, 1, 2, 2]
    got = OT.accept(par, [9, 5, 5, 6, 7, 6], [5, 6, 6, 1, 2, 3], None, [0, 6], [30], [0] * 6, 6)
    assert got == dict(path=[0, 1, 3, -1, -1, -1], count=[3], token=[1], kv_len=[27])
    got = OT.accept(par, [9, 5, 4, 6, 7, 6], [4, 6, 6, 1, 2, 3], None, [0, 6], [30], [0] * 6, 6)
    assert got["path"] == [0, 2, 5, -1, -1, -1] and got["token"] == [3]
    got = OT.accept(par, [9] * 6, [8] * 6, [0], [0, 6], [30], [0] * 6, 6)
    assert got == dict(path=[-1] * 6, count=[0], token=[-1], kv_len=[24])
