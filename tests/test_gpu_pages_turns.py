"""Remaps that drop more entries than the last work group looks at together, without a
launch of their own for the marks: entries marked in several turns and fetched again."""
import os
import re

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_pages import K, check_remap, fresh  # noqa: E402, F401

TEXT = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                         "paper_2608_05483_amd", "csrc", "paged", "pages.hip")).read()


def constant(name):
    return int(re.search(rf"\b{name} = (\d+)[,;]", TEXT).group(1))


CHUNK = constant("kFT")
TURN = CHUNK * constant("kEach")


def drop(K, table, lens, src, keep, page, shares, free, head):
    """check_remap of a call in the form that this file is about."""
    B, most = table.shape
    assert B + len(src) > constant("kInOneRows")
    assert B * most < constant("kMarkShrinking" if len(src) < B else "kMarkAny")
    kept, first = np.zeros(B, int), set()
    for i, b in enumerate(src):
        if 0 <= b < B and b not in first:
            first.add(b)
            n = lens[b] if keep is None else min(lens[b], max(keep[i], 0))
            kept[b] = -(-n // page)
    dropped = -(-np.asarray(lens) // page) - kept
    assert max(dropped[c:c + CHUNK].sum() for c in range(0, B, CHUNK)) > TURN
    return check_remap(K, table, lens, src, keep, page, shares, free, head)


def ended(B, N, on, rng):
    """N new requests of which `on` continue old ones."""
    src = np.full(N, -1)
    src[rng.permutation(N)[:on]] = rng.integers(0, B, on)
    return src


@pytest.mark.parametrize("B,most,N,on", [
    (60, 1000, 60, 8), (60, 1000, 70, 0),      # 30 000 entries, four turns
    (40, 300, 39, 3),                          # a batch that shrinks
    (1100, 58, 1100, 90), (2100, 31, 2200, 5),  # several chunks of requests
])
def test_pages_of_their_own(K, B, most, N, on):
    rng = np.random.default_rng(B + on)
    lens = rng.integers(16 * most * 3 // 4, 16 * most + 1, B)
    table, lens, shares, free, head = fresh(B, most, 16, rng, lens=lens, lead=B * most, spare=90)
    src = ended(B, N, on, rng)
    drop(K, table, lens, src, None, 16, shares, free, head)
    drop(K, table, lens, src, rng.integers(0, 16 * most, N), 16, shares, free, head)
    drop(K, table, lens, src, None, 16, shares, free, head // 7)     # no room for them all


@pytest.mark.parametrize("B,most,times", [(8, 1000, 7), (300, 45, 4)])
@pytest.mark.parametrize("on", [0, 12])
def test_pages_of_several(K, B, most, times, on):
    """Continuations of a request that lie far from each other, in other turns and chunks:
    their pages are dropped by each and put into the list once, or held by who goes on."""
    rng = np.random.default_rng(B + on)
    lens = rng.integers(16 * most * 3 // 4, 16 * most + 1, B)
    table, lens, shares, free, head = fresh(B, most, 16, rng, lens=lens, lead=B * most,
                                            spare=B * times + 90)
    src = np.tile(np.arange(B), times)
    table, lens, shares, free, head, _ = check_remap(K, table, lens, src, None, 16, shares, free,
                                                     head)
    n = len(src)
    _, _, after, _, _, ref = drop(K, table, lens, ended(n, n + 3, on, rng),
                                  rng.integers(0, 16 * most, n + 3), 16, shares, free, head)
    assert ref["meta"][0] > 0 and (after.any() or on == 0)
