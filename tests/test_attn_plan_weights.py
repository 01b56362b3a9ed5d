"""How close a tile's weight is to the keys its steps read, over causal and non-causal
batches with and without windows: the weights divide the work and decide whether a batch
is read tile by tile."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04945_amd", "csrc")
SHIM = r"""
#include <algorithm>
#include "attn_plan.hpp"
using namespace sq;

// Of a batch of one sequence: the largest ratio of a tile's steps to its weight (both in keys), and of all weights
// to all steps and a step more for each tile.  -1: a weight that is not positive.
extern "C" int ratios(int n, int len, int G, int causal, int window, int rows, double* o) {
    const AttnShape a{n, 1, 1, G, len, causal, window, rows, 1, 1, 0};
    const AttnSeq q = attn_seq(a, 0, n, len);
    double heavy = 0, sum = 0, steps = 0;
    int64_t before = 0;
    for (int r = 0; r < q.tiles; ++r) {
        const int64_t w = q.base + q.slope * r;
        if (w <= 0 || attn_before(q, r) != before) return -1;
        before += w;
        const double read = (double)G * kAttnStep * attn_steps(a, q.s, r).count;
        heavy = std::max(heavy, read / w);
        sum += w;
        steps += read + (double)G * kAttnStep;
    }
    if (before != q.weight) return -1;
    o[0] = heavy;
    o[1] = sum / steps;
    return q.tiles;
}

extern "C" int direct(int n, int len, int heads, int G, int causal, int window, int join) {
    AttnShape a = attn_shape(n, 1, heads * G, heads, 128, 1 << 20, causal, window);
    if (join) a.join = join;
    const AttnSeq q = attn_seq(a, 0, n, len);
    int64_t most = 0;
    for (int r = 0; r < q.tiles; ++r) most = std::max(most, (int64_t)G * kAttnStep * attn_steps(a, q.s, r).count);
    const int64_t given = std::max(q.base, q.base + q.slope * (q.tiles - 1));       // as attn_most
    return attn_direct(a, q.weight * heads, given) | attn_direct(a, q.weight * heads, most) << 1;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_plan_weights")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", so],
                   check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("seed", range(100))
def test_weights_are_close_to_the_keys_read(plan, causal, windowed, seed):
    """A weight counts a step more than the tile's keys and a line through them is within a factor of two of what a
    window leaves; steps cover up to two steps more than their keys: a factor of four.  All together weigh at most
    twice what they read (and a step a tile)."""
    rng = random.Random(seed)
    n = rng.choice([1, 30, 500, rng.randint(1, 9000)])
    length = n + rng.choice([0, 0, 100, rng.randint(0, 20000)])
    G = rng.choice([1, 2, 7, 20])
    window = rng.choice([1, 16, 300, 4000, 2 ** 31 - 1, rng.randint(1, length)]) if windowed else 0
    o = (ctypes.c_double * 2)()
    assert plan.ratios(n, length, G, causal, window, rng.choice([16, 32, 128]), o) > 0
    assert o[0] <= 4, ("a tile is longer than its weight", o[0], n, length, G, window)
    assert o[1] <= 2, ("weights without keys", o[1], n, length, G, window)


@pytest.mark.parametrize("n,length,heads,G", [(8192, 8192, 2, 2), (2048, 12048, 2, 5)])
def test_windows_without_a_causal_mask_are_shared_out(plan, n, length, heads, G):
    """Every query sees all later keys: tiles read up to 128 steps, however short the window."""
    assert plan.direct(n, length, heads, G, 0, 16, 0) == 0
