"""Infinities and NaN that a row does see, in caches that are cut into pieces and
prefixes that are shared: every element of the output is of the kind that the
float64 oracle gives (finite, NaN, either infinity), however the step's pieces are
joined."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import BF, HF, G, P, Batch, check  # noqa: E402, F401

SCALE = 0.1


def cell(b, request, key):
    """A key's page and place in it."""
    return int(b.step.table[request, key // b.page]), key % b.page


def check_kinds(b, dt, keys):
    got = b.run(SCALE)
    ref, size = b.ref(SCALE)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(kind(got), kind(ref)), kind.__name__
    fine = np.isfinite(ref)
    ref, size = np.where(fine, ref, 0), np.where(fine & np.isfinite(size), size, 0)
    check(np.where(fine, got, 0), ref, size, dt, keys)
    return got


def spoil(b, request, key, what, value):
    page, at = cell(b, request, key)
    if what == "key":
        b.cache.k[page, :, at] = value
    elif what == "key element":
        b.cache.k[page, :, at, 7] = value
    else:
        b.cache.v[page, :, at, 7] = value


# requests x heads of one token each: up to 1024 rows are joined by four wavefronts, more
# by one
@pytest.mark.parametrize("dt,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("B,H,KH", [(1, 8, 8), (2, 64, 8), (20, 64, 8)])
@pytest.mark.parametrize("what", ["key", "key element", "value"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_decode_in_pieces(G, P, dt, D, B, H, KH, what, value):
    """1537 keys in pieces of 512, the last of one key, which alone is spoilt in the
    first request; a key inside a piece in the last request."""
    b = Batch(G, P, [1536] * B, [1] * B, H, KH, D, dt=dt, seed=B)
    assert b.header()[0] == 4 * B and b.header()[2] > 0
    spoil(b, 0, 1536, what, value)
    if B > 1:
        spoil(b, B - 1, 700, what, value)
    got = check_kinds(b, dt, 1600)
    if what != "value" and math.isnan(value):
        assert np.isnan(got[0]).all()


@pytest.mark.parametrize("B,H,KH", [(1, 8, 8), (20, 64, 8)])
def test_whole_pieces_of_nan(G, P, B, H, KH):
    """All keys of one piece, which then has no maximum; each piece in turn."""
    for piece in range(4):
        b = Batch(G, P, [1536] * B, [1] * B, H, KH, 64, seed=piece)
        for key in range(512 * piece, min(512 * (piece + 1), 1537)):
            spoil(b, 0, key, "key", math.nan)
        assert np.isnan(check_kinds(b, BF, 1600)[0]).all()


@pytest.mark.parametrize("B,H,KH", [(1, 8, 8), (20, 64, 8)])
def test_keys_that_score_minus_infinity(G, P, B, H, KH):
    """A piece, and all pieces, whose scores are all -inf: no weight beside others; a
    row of nothing else is NaN."""
    for last in (512, 1537):
        b = Batch(G, P, [1536] * B, [1] * B, H, KH, 64, seed=last)
        b.q.fill_(0.5)
        for key in range(last):
            spoil(b, 0, key, "key element", -math.inf)
        assert np.isnan(check_kinds(b, BF, 1600)[0]).all() == (last == 1537)


@pytest.mark.parametrize("H,KH,new", [(4, 1, 40), (2, 2, 150)])
@pytest.mark.parametrize("what", ["key", "key element", "value"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_prompts_in_pieces(G, P, H, KH, new, what, value):
    """Tiles over pieces of keys: one old key, which all rows see, and a new one, which
    the later rows do."""
    for key in (300, 2000 + new // 2):
        b = Batch(G, P, [2000], [new], H, KH, seed=new)
        assert b.header()[1] > 1 and b.header()[2] > 0
        spoil(b, 0, key, what, value)
        check_kinds(b, BF, 2200)


@pytest.mark.parametrize("B,H,KH", [(6, 8, 2), (40, 32, 2)])
@pytest.mark.parametrize("what", ["key", "key element", "value"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_shared_prefixes(G, P, B, H, KH, what, value):
    """A key of a prefix, which its members see and the others do not, and a member's
    newest key, which no other sees."""
    for request, key in ((0, 500), (1, None)):
        group = np.arange(B) % 3 - 1
        past = 40 + 5 * (np.arange(B) % 7) + np.where(group >= 0, 1024, 0)
        b = Batch(G, P, past, [1] * B, H, KH, group=group, prefix=[1024, 1024], seed=B)
        request += 1                           # (request 0 is in no group)
        spoil(b, request, int(past[request]) if key is None else key, what, value)
        check_kinds(b, BF, 1200)
