"""Attention rows whose largest weight meets values of zero: the result is made of weights
far below it, whose precision is what the bounds of oracle.attn.attention_bounds allow.

The queries lie along a vector of signs, and so does one key (the sink) of a page of its
own: its logit is `gap` nats, those of the others are about normal."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, ragged, to_device
from gpu_util import dev, host, say
from oracle import attn as A

pytestmark = pytest.mark.gpu

# half a step of a weight below 2^-14, relative to the row's largest
FEW, MANY = 2.0 ** -39, 2.0 ** -36


def sink_batch(page, heads, G, dim, news, lens, gap, ratio, seed):
    """A batch whose sequences hold the sink in their first page, that page's values all zero under a scale `ratio`
    times the others'."""
    rng = np.random.default_rng(seed)
    pages = sum(-(-L // page) for L in lens) + 2
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    sign = rng.choice([-1, 1], dim)
    c.ks[:] = gap / (127 * dim ** 0.5)
    c.vs[:] = rng.uniform(0.01, 0.012, c.vs.shape)
    c.v[:] = rng.integers(60, 128, c.v.shape)
    c.k[:] = np.clip(np.rint(rng.standard_normal(c.k.shape) * (120 / gap)), -127, 127)
    for b in range(len(lens)):
        first = table[b, 0]
        c.k[first, :, 3] = 127 * sign
        c.v[first] = 0
        c.vs[first] *= ratio
    q = (sign * (1 + 0.05 * rng.standard_normal((sum(news), heads * G, dim)))).astype(np.float16)
    return c, q, cu, ln, table


CASES = [
    # page, heads, G, dim, new tokens, lengths, floor
    (64, 1, 1, 128, [1], [131072], FEW),                 # split over waves
    (16, 2, 4, 64, [1, 1], [30000, 500], FEW),
    (32, 1, 2, 128, [15], [20000], FEW),
    (128, 1, 1, 256, [3], [20000], FEW),
    (64, 2, 1, 128, [1, 2], [1000, 900], FEW),           # a workgroup a tile
    (32, 2, 1, 64, [30], [1000], FEW),
    (64, 1, 2, 128, [70], [20000], MANY),                # tiles of 128 rows, split
    (16, 1, 1, 64, [80], [8000], MANY),
    (64, 1, 2, 128, [100], [1000], MANY),                # and whole
    (32, 1, 1, 192, [70], [1000], MANY),
]


@pytest.mark.parametrize("page,heads,G,dim,news,lens,floor", CASES)
@pytest.mark.parametrize("gap,ratio", [(17, 1), (15, 8)])
def test_small_weights_keep_their_precision(page, heads, G, dim, news, lens, floor, gap, ratio):
    c, q, cu, ln, table = sink_batch(page, heads, G, dim, news, lens, gap, ratio, page + dim)
    ref = A.attention(q, c, cu, ln, table, causal=False)
    out, lse = sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), causal=False, want_lse=True)
    d = np.abs(host(out).astype(np.float64) - ref[0])
    bound, _ = A.attention_bounds(*ref, dim, floor)
    say(f"off by {np.linalg.norm(d) / np.linalg.norm(ref[0]):.2e} of the output's norm, "
        f"{(d / bound).max():.2f} of the bound")
    assert (d <= bound).all()
    check_attention(out, ref, (page, dim, gap), lse)


def test_value_scales_of_zero():
    """Values of zero under scales of zero over many keys: zeros, and the logarithm of the sum as the oracle has it."""
    for news in ([1], [70]):
        c, q, cu, ln, table = sink_batch(64, 1, 2, 64, news, [40000], 3, 1, 5)
        c.vs[:], c.v[:] = 0, 0
        ref = A.attention(q, c, cu, ln, table, causal=False)
        out, lse = sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), causal=False, want_lse=True)
        check_attention(out, ref, news, lse)
        assert not host(out).any()
