"""The softmax weights of requests of up to 16 rows a key head count to 16 bits, whether
the request reads its keys alone or shares a prefix with others."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import BF, HF, G, P, Batch, f64, half_step  # noqa: E402, F401

SCALE = 0.25


def one_value(b, ref_rows, dt):
    """The oracle's output with each weight rounded to the type once (of the size it
    has below the row's maximum), as a product of the weights as one value gives it."""
    s = b.step
    table, req, pos = (t.cpu().numpy() for t in (s.table, s.req, s.pos))
    q, k, v = f64(b.q), f64(b.cache.k), f64(b.cache.v)
    r = q.shape[1] // b.KH
    out = np.zeros(q.shape)
    for t in ref_rows:
        idx = np.arange(pos[t] + 1)
        page, off = table[req[t]][idx // b.page], idx % b.page
        for h in range(b.KH):
            x = SCALE * (q[t, h * r:(h + 1) * r] @ k[page, h, off].T)
            p = np.exp(x - x.max(-1, keepdims=True))
            p = f64(torch.from_numpy(p).to(dt))
            out[t, h * r:(h + 1) * r] = p @ v[page, h, off] / p.sum(-1, keepdims=True)
    return out


def check_weights(b, dt):
    """|error| <= the output's rounding and 2^-15 of sum p |v|: queries and keys are
    halves of small whole numbers, so the scores are exact; a weight's two values leave
    2^-16 (fp16 2^-22), its exponent's argument (up to 2^5, three roundings of 2^-24) and
    the exponential 2^-17.4, sums over up to 130 keys 2^-17."""
    g = torch.Generator(device="cuda").manual_seed(7)
    for x in (b.q, b.cache.k):
        x.copy_(torch.randint(-2, 3, x.shape, device="cuda", generator=g) / 2)
    got = b.run(SCALE)
    ref, size = b.ref(SCALE)
    tol = half_step(dt) * np.abs(ref) + 2.0 ** -15 * size
    assert (np.abs(got - ref) <= tol).all()
    # (weights of one value each would not pass)
    assert (np.abs(one_value(b, range(len(ref)), dt) - ref) > tol).mean() > 0.01


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 128), (BF, 64), (HF, 64)])
@pytest.mark.parametrize("H,KH,new", [(2, 2, 1), (4, 1, 4), (16, 1, 1)])
def test_alone(G, P, dt, D, H, KH, new):
    past = [9, 30, 63, 100, 125]
    check_weights(Batch(G, P, past, [new] * 5, H, KH, D, dt=dt, seed=D), dt)


@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 128), (BF, 64), (HF, 64)])
@pytest.mark.parametrize("B,H,KH,new", [(3, 4, 1, 1), (24, 4, 1, 1), (40, 8, 2, 1), (30, 2, 1, 5)])
def test_behind_a_shared_prefix(G, P, dt, D, B, H, KH, new):
    """A prefix that few rows share, and one that fills tiles."""
    past = 64 + np.arange(B) % 30
    b = Batch(G, P, past, [new] * B, H, KH, D, dt=dt, group=[0] * B, prefix=[64], seed=D)
    assert (b.header()[1] > 0) == (B * new * H // KH > 16)
    check_weights(b, dt)
