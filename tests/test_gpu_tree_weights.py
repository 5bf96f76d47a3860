"""The softmax weights of plora_attn_tree count to as many bits as plora_attn_paged's: to
16 over the keys of requests of up to 16 rows a key head, and over prefixes that requests
of any size share."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tree as OT  # noqa: E402
from test_gpu_paged import BF, HF, G, P, check, f64, half_step  # noqa: E402, F401
from test_gpu_tree import R, TreeBatch, host  # noqa: E402, F401

SCALE = 0.25
TYPES = [(BF, 128), (HF, 128), (BF, 64), (HF, 64)]


def one_value(b, dt):
    """The oracle's output with each weight rounded to the type once (of the size it has
    below the row's maximum)."""
    table, s = b.step.table.cpu().numpy(), host(b.step)
    q, k, v = f64(b.q), f64(b.cache.k), f64(b.cache.v)
    r = q.shape[1] // b.KH
    out = np.zeros(q.shape)
    for i in range(len(s["kv_len"])):
        at = OT.rows(s["q_start"], s["req"], i)
        past = int(s["kv_len"][i]) - len(at)
        for t, way in zip(at, OT.paths([int(b.parent[t]) for t in at])):
            idx = np.concatenate([np.arange(past), past + np.array(way)])
            page, off = table[i][idx // b.page], idx % b.page
            for h in range(b.KH):
                x = SCALE * (q[t, h * r:(h + 1) * r] @ k[page, h, off].T)
                p = f64(torch.from_numpy(np.exp(x - x.max(-1, keepdims=True))).to(dt))
                out[t, h * r:(h + 1) * r] = p @ v[page, h, off] / p.sum(-1, keepdims=True)
    return out


def check_weights(b, dt, prefix_only=False):
    """|error| <= the output's rounding and 2^-15 of sum p |v|: queries and keys are halves
    of small whole numbers, so the scores are exact; a weight's two values leave 2^-16
    (fp16 2^-22), its exponent's argument (up to 2^5, three roundings of 2^-24) and the
    exponential 2^-17.4, sums over up to 160 keys 2^-17.  prefix_only: the new keys score
    40 less than the others' scale of 1.4, so that all of a row's weight is the prefix's
    (theirs is below 2^-40, however it is rounded)."""
    g = torch.Generator(device="cuda").manual_seed(7)
    for x in (b.q, b.cache.k):
        x.copy_(torch.randint(-2, 3, x.shape, device="cuda", generator=g) / 2)
    if prefix_only:
        slot = b.step.slot
        b.q[:, :, 0] = 2.0
        b.cache.k[:, :, :, 0] = 0.0
        b.cache.k[slot // b.page, :, slot % b.page, 0] = -80.0
    got = b.run(SCALE)
    ref, size = b.ref(SCALE)
    tol = half_step(dt) * np.abs(ref) + 2.0 ** -15 * size
    assert (np.abs(got - ref) <= tol).all()
    # (weights of one value each would not pass)
    assert (np.abs(one_value(b, dt) - ref) > tol).mean() > 0.01


@pytest.mark.parametrize("dt,D", TYPES)
@pytest.mark.parametrize("H,KH,new", [(2, 2, 7), (4, 1, 4), (16, 1, 1)])
def test_alone(G, P, R, dt, D, H, KH, new):
    past = [9, 30, 63, 100, 125]
    check_weights(TreeBatch(G, P, R, past, [new] * 5, H, KH, D, dt=dt, seed=D), dt)


# tokens by request, heads over key heads
GROUPS = [([1, 4, 3], 4, 1),                   # few rows together
          ([3, 2, 4] * 8, 4, 1),               # small requests, which fill tiles
          ([3, 7, 5, 4], 8, 1),                # larger ones alone
          ([30, 64, 9], 4, 2),
          ([3, 7, 1, 16, 5, 2], 8, 1)]         # both


@pytest.mark.parametrize("dt,D", TYPES)
@pytest.mark.parametrize("new,H,KH", GROUPS)
def test_behind_a_shared_prefix(G, P, R, dt, D, new, H, KH):
    B = len(new)
    b = TreeBatch(G, P, R, [64] * B, new, H, KH, D, dt=dt, group=[0] * B, prefix=[64], seed=D)
    assert (b.header()[1] > 0) == (sum(new) * H // KH > 16)
    check_weights(b, dt, prefix_only=True)


@pytest.mark.parametrize("dt,D", TYPES)
@pytest.mark.parametrize("new,H,KH", GROUPS)
def test_chains_behind_a_shared_prefix_are_causal(G, P, R, dt, D, new, H, KH):
    """The bits of plora_attn_paged, whoever shares the prefix."""
    B = len(new)
    past = 700 + 5 * np.arange(B)
    b = TreeBatch(G, P, R, past, new, H, KH, D, dt=dt, group=[0] * B, prefix=[650], seed=B,
                  kinds=("chain",))
    G.attn_paged(b.q, b.cache, b.step, b.plan, 0.1, b.out)
    torch.cuda.synchronize()
    want = f64(b.out)
    b.out.fill_(3)
    assert np.array_equal(b.run(0.1), want)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("n", [5, 90])
def test_a_tree_that_looks_like_a_chain_is_none(G, P, R, D, n):
    """Every parent the node before but one: that node, and those behind it, do not see
    the node that is passed over."""
    b = TreeBatch(G, P, R, [40], [n], 4, 2, D, kinds=("chain",), seed=n)
    chain = b.run(0.1)
    b.parent[3] = 1
    R.tree_plan(torch.from_numpy(b.parent).int().cuda(), b.step, b.tree)
    got = b.run(0.1)
    assert b.tree.info[0].tolist() == [1, 0]
    check(got, *b.ref(0.1), BF, 200)
    assert (got[3:] != chain[3:]).any(-1).all()
