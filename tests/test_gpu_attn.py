"""Attention over the paged 8-bit cache against the oracle in fp64, within bounds
derived from the arithmetic (oracle.attn.attention_bounds): masks, head layouts, page
sizes, ragged batches, rows that see nothing, values that must not leak."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, normal, ragged, strided, to_device
from gpu_util import assert_bits, dev, host, say
from oracle import attn as A

pytestmark = pytest.mark.gpu


def run(page, heads, G, dim, news, lens, causal=True, window=0, seed=0, scale=None, lead=0, extra=0, q_scale=1.0,
        change=None):
    rng = np.random.default_rng(seed + page + dim + G)
    pages = sum(-(-L // page) for L in lens) + 2
    max_pages = max(-(-L // page) for L in lens) + extra
    cu, ln, table = ragged(news, lens, max(1, max_pages), page, pages, rng, lead)
    c = filled_cache(pages, heads, dim, page, rng)
    T = sum(news) + lead + 1
    q = normal(rng, T, heads * G, dim, scale=q_scale)
    if change:
        change(c, table, rng)
    out = torch.full((T, heads * G, dim), 9.0, dtype=torch.float16, device="cuda")
    lse = torch.full((T, heads * G), 9.0, dtype=torch.float32, device="cuda")
    got = sq.attn_kv8(strided(q), to_device(c), dev(cu), dev(ln), dev(table), causal=causal, window=window, scale=scale,
                      out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    ref = A.attention(q, c, cu, ln, table, causal, window, scale)
    worst = check_attention(out, ref, (page, heads, G, dim, news, lens), lse)
    rest = np.setdiff1d(np.arange(T), np.r_[cu[0]:cu[-1]])
    assert (host(out)[rest] == 9).all() and (host(lse)[rest] == 9).all()      # rows of no sequence
    return worst


SHAPES = [
    # page, heads, G, dim, new tokens, lengths
    (64, 1, 1, 128, [1], [1]),
    (16, 2, 1, 64, [1, 1, 1], [1, 17, 63]),
    (64, 4, 7, 128, [1, 1, 1, 1], [64, 65, 700, 3]),
    (128, 2, 8, 128, [1], [1500]),
    (32, 2, 5, 80, [1, 1], [333, 64]),
    (16, 3, 4, 96, [3, 1, 9], [50, 128, 9]),
    (64, 1, 16, 256, [1, 2], [130, 200]),
    (128, 2, 20, 48, [1, 1], [257, 90]),                # more query heads to a key head than a tile has rows
    (64, 2, 2, 128, [40, 1, 0, 17], [40, 400, 30, 100]),
    (32, 4, 1, 128, [33], [200]),
    (16, 1, 3, 16, [70], [70]),
    (64, 2, 1, 64, [300], [320]),
    (64, 1, 7, 128, [150, 90], [150, 500]),
]


@pytest.mark.parametrize("page,heads,G,dim,news,lens", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(page, heads, G, dim, news, lens, causal):
    worst = run(page, heads, G, dim, news, lens, causal, lead=1)
    say(f"largest error {worst:.2f} of its bound")


@pytest.mark.parametrize("page,heads,G,dim,news,lens", [s for s in SHAPES if max(s[5]) > 40][::2])
@pytest.mark.parametrize("window", [1, 20, 64, 1000])
@pytest.mark.parametrize("causal", [True, False])
def test_window(page, heads, G, dim, news, lens, window, causal):
    run(page, heads, G, dim, news, lens, causal, window)


def test_rows_that_see_nothing():
    """Empty caches, lengths below the number of new tokens, a table of no pages: zeros, lse -inf."""
    run(64, 2, 2, 64, [3, 5, 2, 130], [0, 2, 2, 1])
    run(64, 2, 2, 64, [3, 5, 2, 130], [0, 2, 2, 1], causal=False)

    def none(c, table, rng):
        table[:] = -1
    run(16, 2, 3, 128, [2, 40], [40, 40], change=none)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_missing_pages_are_masked(page):
    def holes(c, table, rng):
        table[0, 1] = -1
        table[1, 0] = c.pages
        table[2, 2] = 2 ** 31 - 1
    for news in ([1, 1, 1], [9, 60, 130]):
        run(page, 2, 4, 64, news, [4 * page - 3, 3 * page, 5 * page], change=holes)


@pytest.mark.parametrize("news", [[1, 1], [20, 70]])
def test_no_leak_from_masked_places(news):
    """Codes past the length, pages of no one, and pages wholly outside the window hold the worst values
    (largest codes, infinite and NaN scales) and change nothing."""
    page, heads, G, dim = 16, 2, 4, 64
    rng = np.random.default_rng(8)
    lens = [205, 100]
    cu, ln, table = ragged(news, lens, 20, page, 40, rng)
    c = filled_cache(40, heads, dim, page, rng)
    q = normal(rng, sum(news), heads * G, dim)
    for window in (0, 17):
        ref = A.attention(q, c, cu, ln, table, True, window)
        bad = c.copy()
        used = set()
        for b, L in enumerate(lens):
            first = max(0, L - news[b] - window + 1) // page if window else 0
            used |= {int(p) for p in table[b, first:-(-L // page)]}
            if L % page:
                pid = table[b, L // page]
                bad.k[pid, :, L % page:] = -128
                bad.v[pid, :, :, L % page:] = 127
        for pid in set(range(40)) - used:
            bad.k[pid], bad.v[pid] = 127, -128
            bad.ks[pid], bad.vs[pid] = np.inf, np.nan
        bad_table = table.copy()
        for b, L in enumerate(lens):
            bad_table[b, -(-L // page):] = next(iter(set(range(40)) - used))
        out, lse = sq.attn_kv8(dev(q), to_device(bad), dev(cu), dev(ln), dev(bad_table), window=window, want_lse=True)
        check_attention(out, ref, window, lse)


@pytest.mark.parametrize("news", [[1], [70]])
def test_scales_of_any_size(news):
    """Value scales over twelve orders of magnitude, a zero one, large and small logits."""
    def spread(c, table, rng):
        c.vs[:] = (10.0 ** rng.uniform(-9, 2.0, c.vs.shape)).astype(np.float32)
        c.vs[table[0, 2]] = 0
        c.ks[table[0, 1]] = 0
    for q_scale in (1e-3, 1.0, 30.0):
        run(16, 2, 4, 64, news, [150], change=spread, q_scale=q_scale)


def test_scale_argument_and_extreme_codes():
    def extreme(c, table, rng):
        c.k[:], c.v[:] = -128, 127
        c.ks[:], c.vs[:] = 0.02, 0.02
    run(64, 2, 2, 128, [1, 30], [100, 200], change=extreme)
    run(64, 2, 2, 128, [1, 30], [100, 200], scale=0.0)
    run(64, 2, 2, 128, [1, 30], [100, 200], scale=-0.3)


@pytest.mark.parametrize("extra", [0, 1000])
def test_split_over_many_workers(extra):
    """A few long rows, joined from partial results; a table much wider than the lengths."""
    run(64, 2, 4, 64, [1, 1], [5000, 70], extra=extra)
    run(128, 1, 1, 128, [2], [3000], causal=False, extra=extra)
    run(64, 2, 4, 64, [64, 1], [2000, 70], extra=extra)


def test_many_sequences():
    """More sequences than a wave has lanes, most of them short, some without new tokens."""
    rng = np.random.default_rng(9)
    lens = rng.integers(1, 90, 150).tolist()
    lens[77] = 2000
    news = [0 if b % 9 == 4 else 1 for b in range(150)]
    run(32, 2, 2, 64, news, lens)
    news = [0 if b % 9 == 4 else min(L, 1 + b % 7) for b, L in enumerate(lens)]
    run(32, 2, 2, 64, news, lens)


def test_deterministic_and_workspace():
    """Two calls, on a workspace of all ones and on one of the exact size, give the same bits."""
    rng = np.random.default_rng(10)
    c = filled_cache(80, 4, 128, 64, rng)
    cu, ln, table = ragged([1, 3], [3000, 1500], 47, 64, 80, rng)
    q = dev(normal(rng, 4, 28, 128))
    cache, cu, ln, table = to_device(c), dev(cu), dev(ln), dev(table)
    need = sq.attn_kv8_workspace_bytes(4, 2, 28, 4, 128, 47 * 64)
    a = host(sq.attn_kv8(q, cache, cu, ln, table))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    assert_bits(host(sq.attn_kv8(q, cache, cu, ln, table, ws=ws)), a, "workspace of NaN")
    assert need > 0
    with pytest.raises(sq.StarQuantError, match="workspace"):
        sq.attn_kv8(q, cache, cu, ln, table, ws=ws[:need - 256])


def test_empty_batches():
    rng = np.random.default_rng(11)
    cache = to_device(filled_cache(2, 2, 32, 16, rng))
    z = torch.zeros(0, 4, 32, dtype=torch.float16, device="cuda")
    cu0, l0 = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    assert sq.attn_kv8(z, cache, cu0, l0, torch.zeros(0, 3, dtype=torch.int32, device="cuda")).shape == (0, 4, 32)
    q = dev(normal(rng, 2, 4, 32))
    cu, ln = dev(np.array([0, 2], np.int32)), dev(np.array([5], np.int32))
    out, lse = sq.attn_kv8(q, cache, cu, ln, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), want_lse=True)
    assert not host(out).any() and np.isneginf(host(lse)).all()               # a table without room
