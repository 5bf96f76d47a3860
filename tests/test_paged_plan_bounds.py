"""The caps of the attention plan's items and partial rows (bounds in attn_plan.h, compiled
here for the host) hold for any lengths, and are what the library's sizes are made of."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paged_plan_model as M
from paper_2608_05483_amd import build as B
from paper_2608_05483_amd import paged as G

SHIM = """
#include "attn_plan.h"
extern "C" void caps(const plora_attn_shape* s, int64_t* out) {
  const paged::Bounds b = paged::bounds(*s);
  out[0] = b.few_cap, out[1] = b.tile_cap, out[2] = b.part_rows;
  out[3] = sizeof(paged::Item), out[4] = sizeof(paged::ReqInfo);
  out[5] = paged::kHere, out[6] = paged::kKeptArrays;
}
"""


@pytest.fixture(scope="module")
def caps(tmp_path_factory):
    d = tmp_path_factory.mktemp("shim")
    src, out = str(d / "shim.hip"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run([B.HIPCC, "--offload-host-only", *B.CFLAGS, "-shared", src, "-o", out],
                   check=True, capture_output=True)
    lib = ctypes.CDLL(out)

    def f(shape):
        a = (ctypes.c_int64 * 7)()
        lib.caps(ctypes.byref(shape), a)
        return list(a)
    return f


def shape_of(new, T, H, KH, max_q, shared, D=128):
    return G.plora_attn_shape(len(new), T, H, KH, D, max_q, int(shared), 0)


def holds(caps, past, new, H, KH, page=16, group=None, prefix=(), pad=0, slack=0):
    sh = shape_of(new, int(np.sum(new)) + pad, H, KH, int(np.max(new)) + slack, group is not None)
    few_cap, tile_cap, part_rows = caps(sh)[:3]
    few, tiles, parts, _, _, later = M.plan(M.sets_of(past, new, H // KH, page, group, prefix), KH)
    assert few + later <= few_cap and tiles <= tile_cap and parts <= part_rows, \
        (past, new, H, KH, group, prefix)


def test_random_steps(caps):
    rng = np.random.default_rng(11)
    for _ in range(400):
        B = int(rng.integers(1, 80))
        KH = int(rng.choice([1, 2, 3, 8, 32, 100]))
        H = KH * int(rng.choice([1, 3, 8, 16, 20]))
        new = rng.integers(0, int(rng.choice([1, 2, 9, 400])) + 1, B)
        new[0] = max(new[0], 1)
        past = rng.integers(0, int(rng.choice([1, 500, 20000, 2000000])) + 1, B)
        group = prefix = None
        if rng.random() < 0.6:
            n = int(rng.integers(1, 9))
            prefix = rng.integers(0, int(rng.choice([100, 9000])), n)
            group = rng.integers(-1, n, B)
            past = past + np.where(group >= 0, prefix[group], 0)
        holds(caps, past, new, H, KH, int(rng.choice([16, 64, 256])), group,
              prefix if group is not None else (), int(rng.integers(0, 5)), int(rng.integers(0, 3)))


@pytest.mark.parametrize("H,KH", [(1, 1), (17, 1), (16, 1), (129, 1), (8, 8), (128, 128)])
def test_steps_at_the_edges(caps, H, KH):
    """One token or one tile more than fits, pieces of one key, groups of two."""
    for B in (1, 2, 3, 64):
        for past in (0, 1, 511, 512, 513, 1024, 1537, 100000):
            for n in (1, 2, 8, 16, 17, 127, 129):
                new = np.full(B, n)
                holds(caps, np.full(B, past), new, H, KH)
                group = np.arange(B) // 2
                holds(caps, np.full(B, past), new, H, KH, 16, group, np.full(B, past))
                holds(caps, np.full(B, past), new, H, KH, 16, np.zeros(B, int), [past])


def test_sizes_follow_the_bounds(caps):
    """The plan's and the workspace's bytes: header, items, gathered tokens, requests, and
    what is kept of many requests; maxima, sums and outputs of the partial rows."""
    up = lambda n: (n + 255) // 256 * 256
    for B, T, H, KH, D, max_q, shared in [
            (1, 1, 8, 8, 128, 1, 0), (64, 64, 32, 32, 64, 1, 0), (1024, 3000, 16, 2, 128, 40, 1),
            (1025, 3000, 16, 2, 128, 40, 1), (5, 9000, 20, 1, 64, 5000, 0)]:
        sh = G.plora_attn_shape(B, T, H, KH, D, max_q, shared, 0)
        few, tile, rows, item, info, here, arrays = caps(sh)
        assert G.attn_plan_bytes(sh) == 256 + up(few * item) + up(tile * item) + \
            up(4 * T if shared else 0) + up(B * info) + up((B + 1) * arrays * 4 if B > here else 0)
        n = rows * KH
        assert G.attn_paged_workspace_bytes(sh) == 2 * up(4 * n) + up(4 * n * D)
