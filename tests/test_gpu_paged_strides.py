"""Pools whose keys lie far apart: offsets inside a page that pass 32 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import paged as OP  # noqa: E402
from test_gpu_paged import BF, G, P, check, f64, i32  # noqa: E402, F401


@pytest.mark.parametrize("page,stride", [(256, 9 << 20), (128, 20 << 20), (256, (1 << 25) - 8)])
def test_keys_far_apart(G, P, page, stride):
    """A pool in the order [key of the page][page][head][dim] whose last keys begin
    more than 2^31 elements behind the first, up to the longest token stride: what
    rope_append stores there, attention reads, for few rows and for tiles."""
    n_pages, KH, H, D = 5, 2, 8, 128
    assert (page - 1) * stride > 2 ** 31
    torch.cuda.empty_cache()
    size = (page - 1) * stride + n_pages * KH * D
    pool = lambda: torch.empty(size, dtype=BF, device="cuda").as_strided(
        (n_pages, KH, page, D), (KH * D, D, stride, 1))
    k, v = pool(), pool()
    g = torch.Generator(device="cuda").manual_seed(page)
    mk = lambda *s: torch.randn(s, device="cuda", generator=g).to(BF)
    k.copy_(mk(n_pages, KH, page, D)), v.copy_(mk(n_pages, KH, page, D))
    cache = G.KVCache(k, v)
    table = np.array([[3, 1], [4, 0]])
    step = G.Step(2, 31, page, 2, table=i32(table))
    G.kv_plan(i32([page + 100, page - 11]), i32([1, 30]), i32([0]), i32([0]), i32([0]), step)
    q, kk, vv = mk(31, H, D), mk(31, KH, D), mk(31, KH, D)
    out = torch.zeros_like(q)
    plan = G.AttnPlan(step, H, KH, D, max_q=30)
    G.attn_plan(step, plan)
    G.run_layers(step, plan, [(q, kk, vv, cache, out)], G.rope_turns(D), 0.1)
    torch.cuda.synchronize()
    slot = step.slot.cpu().numpy()
    assert (slot >= 0).all()
    for t, s in enumerate(slot):
        assert torch.equal(v[s // page, :, s % page], vv[t])
    ref, size = OP.attention(f64(q), f64(k), f64(v), table, None, None, step.req.cpu().numpy(),
                             step.pos.cpu().numpy(), page, 0.1)
    check(f64(out), ref, size, BF, 400)
