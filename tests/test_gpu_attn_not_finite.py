"""What is not finite reaches the rows that meet it, as NaN, and no others: scales of
visible pages (an overflow upstream, or a page that was never written), and queries whose
products are all -inf."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, normal, ragged, to_device
from gpu_util import dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu

FORMS = [
    # page, heads, G, dim, new tokens, lengths
    (64, 2, 4, 64, [3, 2], [200, 70]),                   # tiles of 16
    (16, 2, 4, 128, [2, 3], [200, 70]),
    (16, 2, 1, 64, [1, 1], [5000, 40]),                  # split over waves
    (128, 1, 2, 256, [3], [3000]),
    (32, 2, 1, 128, [30, 20], [100, 200]),               # tiles of 32
    (64, 1, 2, 128, [90, 70], [150, 300]),               # tiles of 128
    (32, 2, 1, 128, [90, 70], [150, 300]),
    (16, 1, 1, 192, [100], [170]),
    (64, 2, 4, 64, [70, 30], [3000, 100]),               # split
    (32, 1, 2, 80, [90], [2500]),
]


def seen_pages(b, i, h, cu, ln, page, causal, window):
    """Entries of sequence b's table that its new token i sees keys of."""
    n, L = int(cu[b + 1] - cu[b]), int(ln[b])
    p = L - n + i
    lo, hi = max(0, p - window + 1) if window else 0, min(L, p + 1) if causal else L
    return range(lo // page, -(-hi // page)) if hi > lo else ()


@pytest.mark.parametrize("page,heads,G,dim,news,lens", FORMS)
@pytest.mark.parametrize("which,value", [("ks", np.nan), ("ks", np.inf), ("ks", -0.01), ("vs", np.nan), ("vs", np.inf),
                                         ("vs", -np.inf)])
def test_scales_that_are_not(page, heads, G, dim, news, lens, which, value):
    rng = np.random.default_rng(page + dim)
    pages = sum(-(-L // page) for L in lens) + 2
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    q = normal(rng, sum(news), heads * G, dim)
    bad = c.copy()
    last = -(-lens[0] // page) - 1
    spoiled = {(0, last): heads - 1, (0, 1): 0}          # the new tokens' page, and an old one: of one head each
    for (b, j), h in spoiled.items():
        (bad.ks if which == "ks" else bad.vs)[table[b, j], h] = value
    for causal, window in ((True, 0), (False, 0), (True, 20), (False, 33)):
        out, lse = (host(t) for t in sq.attn_kv8(dev(q), to_device(bad), dev(cu), dev(ln), dev(table), causal=causal,
                                                 window=window, want_lse=True))
        ref = A.attention(q, c, cu, ln, table, causal, window)
        hit = 0
        for b in range(len(lens)):
            for i in range(news[b]):
                for h in range(heads * G):
                    js = seen_pages(b, i, h, cu, ln, page, causal, window)
                    if any(spoiled.get((b, j)) == h // G for j in js):
                        t = int(cu[b]) + i
                        assert np.isnan(out[t, h]).all() and np.isnan(lse[t, h]), (t, h, causal, window)
                        out[t, h], lse[t, h] = ref[0][t, h], ref[1][t, h]
                        hit += 1
        assert hit
        check_attention(dev(out), ref, (causal, window), dev(lse))


def test_scale_of_minus_zero():
    rng = np.random.default_rng(1)
    c = filled_cache(4, 1, 64, 64, rng)
    cu, ln, table = ragged([2], [150], 3, 64, 4, rng)
    c.ks[table[0, 0]], c.vs[table[0, 1]] = -0.0, -0.0
    q = normal(rng, 2, 2, 64)
    out, lse = sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), want_lse=True)
    check_attention(out, A.attention(q, c, cu, ln, table), 0, lse)


@pytest.mark.parametrize("page,heads,G,dim,news,lens", FORMS)
def test_products_of_minus_infinity(page, heads, G, dim, news, lens):
    """An infinite query against codes of the other sign: every product is -inf, the row NaN; one that sees no key
    stays zeros and lse -inf."""
    rng = np.random.default_rng(page + dim)
    pages = sum(-(-L // page) for L in lens) + 2
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    ln[-1] = max(1, news[-1] - 1)                        # the last sequence's first token sees none
    c = filled_cache(pages, heads, dim, page, rng)
    c.k[..., 5] = np.maximum(1, np.abs(c.k[..., 5].astype(np.int16)))
    q = normal(rng, sum(news), heads * G, dim)
    bad = q.copy()
    rows = [(0, 0), (sum(news) - 1, heads * G - 1), (int(cu[-2]), 0)]
    for t, h in rows:
        bad[t, h, 5] = -np.inf
    ref = A.attention(q, c, cu, ln, table)
    out, lse = (host(t) for t in sq.attn_kv8(dev(bad), to_device(c), dev(cu), dev(ln), dev(table), want_lse=True))
    for t, h in rows:
        if np.isfinite(ref[1][t, h]):
            assert np.isnan(out[t, h]).all() and np.isnan(lse[t, h]), (t, h)
            out[t, h], lse[t, h] = ref[0][t, h], ref[1][t, h]
    check_attention(dev(out), ref, news, dev(lse))
