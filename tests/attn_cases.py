"""Inputs of the rotary, cache and attention tests, and their comparisons."""
import numpy as np
import torch

import paper_2606_04945_amd as sq
from gpu_util import dev, host
from oracle import attn as A


def ragged(news, lens, max_pages, page, pages, rng, lead=0):
    """cu, lens and a table of shuffled distinct pages; entries past a length are no pages."""
    cu = lead + np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    order = iter(rng.permutation(pages))
    table = np.full((len(lens), max_pages), -7, np.int32)
    for b, L in enumerate(lens):
        for j in range(-(-L // page)):
            table[b, j] = next(order)
    return cu, np.array(lens, np.int32), table


def filled_cache(pages, heads, dim, page, rng):
    c = A.Cache(pages, heads, dim, page)
    c.k = rng.integers(-127, 128, c.k.shape).astype(np.int8)
    c.v = rng.integers(-127, 128, c.v.shape).astype(np.int8)
    c.ks = rng.uniform(0.005, 0.03, c.ks.shape).astype(np.float32)
    c.vs = rng.uniform(0.005, 0.03, c.vs.shape).astype(np.float32)
    return c


def to_device(c):
    return sq.KVCache(dev(c.k), dev(c.v), dev(c.ks), dev(c.vs))


def normal(rng, *shape, scale=1.0):
    return (rng.standard_normal(shape) * scale).astype(np.float16)


def strided(a, heads_before=1, heads_after=2):
    """a [T, H, D] as a view into wider rows on the device (a fused projection's output)."""
    T, H, D = a.shape
    wide = torch.full((T, heads_before + H + heads_after, D), 77.0, dtype=torch.float16, device="cuda")
    wide[:, heads_before:heads_before + H] = dev(a)
    return wide[:, heads_before:heads_before + H]


def check_attention(got, ref, what, lse=None, rows=None):
    out, rlse, e = ref
    rows = np.isfinite(out[:, 0, 0]) if rows is None else rows
    D = out.shape[2]
    b_out, b_lse = A.attention_bounds(out, rlse, e, D)
    g = host(got).astype(np.float64) if isinstance(got, torch.Tensor) else got.astype(np.float64)
    d = np.abs(g - out)[rows]
    worst = (d / b_out[rows]).max(initial=0.0)
    assert np.isfinite(g[rows]).all() and worst <= 1, (what, worst)
    if lse is not None:
        gl = host(lse).astype(np.float64)[rows]
        rl = rlse[rows]
        assert np.array_equal(np.isinf(gl), np.isinf(rl)), what
        fin = np.isfinite(rl)
        assert (np.abs(gl[fin] - rl[fin]) <= b_lse[rows][fin]).all(), (what, np.abs(gl[fin] - rl[fin]).max())
    return worst
