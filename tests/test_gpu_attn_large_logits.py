"""Attention whose logits are far from zero, of either sign: a hard maximum.

Queries of ones, integer codes and scales that are powers of two: every logit is an exact
integer times a power of two (and log2 e, one rounding that keeps their order), so that the
largest of a row is the oracle's, its weight 1 and every other 0."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import filled_cache, ragged, to_device
from gpu_util import dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads,G,dim,news,lens", [
    (64, 2, 3, 64, [1, 2], [200, 70]),                   # tiles of 16, a workgroup a tile
    (16, 1, 2, 128, [1, 1], [5000, 90]),                 # split over waves
    (32, 1, 1, 256, [4], [300]),
    (32, 2, 1, 128, [30], [300]),                        # tiles of 32
    (64, 2, 2, 128, [80, 50], [300, 50]),                # tiles of 128
    (16, 1, 2, 64, [100], [170]),
    (64, 1, 4, 128, [40, 30], [4000, 30]),               # split
])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("power", [7, 20, 37, 60, 90])
def test_hard_maximum(page, heads, G, dim, news, lens, sign, power):
    rng = np.random.default_rng(page + dim + power)
    pages = sum(-(-L // page) for L in lens) + 2
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    c.k[:] = sign * rng.integers(1, 128, c.k.shape)
    c.ks[:], c.vs[:] = 0.5, 0.01
    q = np.ones((sum(news), heads * G, dim), np.float16)
    for kw in (dict(causal=True), dict(causal=False), dict(causal=True, window=40)):
        scale = 2.0 ** power
        out, lse, _ = A.attention(q, c, cu, ln, table, scale=scale, **kw)
        o, z = (host(t).astype(np.float64)
                for t in sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), scale=scale, want_lse=True, **kw))
        # two roundings to fp16 (weights that tie, and the result), a few in fp32
        assert (np.abs(o - out) <= 2.0 ** -10 * np.abs(out) + 2.0 ** -18).all(), kw
        assert (np.abs(z - lse) <= 2.0 ** -21 * np.abs(lse)).all(), kw
