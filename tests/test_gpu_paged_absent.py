"""rope_append with nothing to turn in q, or nothing to store."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import BF, G, P, i32  # noqa: E402, F401


@pytest.mark.parametrize("H,KH", [(0, 2), (3, 0), (0, 0)])
def test_rope_append_without_q_or_without_keys(G, P, H, KH):
    """What is there is as in a call that has both."""
    T, D, page = 9, 64, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda n: torch.randn((T, n, D), device="cuda", generator=g).to(BF)
    q, k, v = mk(3), mk(2), mk(2)
    pos, turns = i32(np.arange(T) * 37), G.rope_turns(D)
    slot = torch.arange(T, device="cuda") + 11
    both = G.KVCache.empty(2, page, 2, D)
    want = torch.zeros_like(q)
    G.rope_append(q, k, v, pos, slot, turns, both, want)
    cache, out = G.KVCache.empty(2, page, KH, D), torch.zeros_like(q[:, :H])
    G.rope_append(q[:, :H], k[:, :KH], v[:, :KH], pos, slot, turns, cache, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want[:, :H])
    assert torch.equal(cache.k, both.k[:, :KH]) and torch.equal(cache.v, both.v[:, :KH])
    assert KH == 0 or (cache.k.abs().amax((1, 3)) > 0).sum() == T
