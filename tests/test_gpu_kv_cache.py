"""The paged 8-bit cache against the oracle: append (scales, codes, requantisation,
rotation) and reading back.

Without rotation everything is bit-exact: fp32 scales and codes are fixed by the
interface.  Rotated keys are within 2^-20 of their page's absmax (each component's
|u| + |v| is at most twice the larger of the rotated pair), so scales are within
2^-20 relative and a code is rint of a quotient off by at most 127 2^-19."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import filled_cache, normal, ragged, strided, to_device
from gpu_util import assert_bits, dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


def same_cache(got, want, what):
    for name, x, y in zip(("k", "v", "k_scale", "v_scale"), got, (want.k, want.v, want.ks, want.vs)):
        assert_bits(host(x), y, f"{what}: {name}")


BATCHES = [
    # page, heads, dim, new tokens, lengths
    (16, 1, 16, [1], [1]),
    (64, 4, 128, [1, 1, 1], [64, 65, 200]),                       # a page's last slot, first slot, inside
    (64, 2, 128, [130, 0, 7, 64], [130, 50, 70, 128]),            # whole pages, none new, ragged
    (32, 3, 80, [31, 33, 1], [31, 64, 33]),
    (128, 2, 256, [129, 5], [140, 127]),
    (16, 8, 64, [200, 16, 15], [207, 16, 31]),
    (16, 2, 48, [5, 3], [3, 0]),                                  # lengths below the number of new tokens
]


@pytest.mark.parametrize("page,heads,dim,news,lens", BATCHES)
def test_append_bit_exact(page, heads, dim, news, lens):
    rng = np.random.default_rng(page + dim)
    T = sum(news) + 5
    pages = sum(-(-L // page) for L in lens) + 3
    cu, ln, table = ragged(news, lens, max(1, max(-(-L // page) for L in lens)), page, pages, rng, lead=2)
    want = filled_cache(pages, heads, dim, page, rng)
    cache = to_device(want)
    K, V = normal(rng, T, heads, dim), normal(rng, T, heads, dim, scale=2)
    K[::3] *= np.float16(4)                                       # some pages' scales grow, some do not
    args = (strided(K), strided(V, 2, 0), dev(cu), dev(ln), dev(table))
    assert sq.kv_append(cache, *args) is None
    A.append(want, K.astype(np.float32), V.astype(np.float32), cu, ln, table)
    same_cache(cache, want, "first")
    sq.kv_append(cache, *args)                                    # the same call again changes nothing
    same_cache(cache, want, "again")
    pids = np.arange(-1, pages + 1).astype(np.int32)
    k, v = sq.kv_read(cache, dev(pids))
    rk, rv = A.values(want, pids)
    # code times scale in fp32, one rounding to fp16: the product of an 8-bit integer and an fp32 rounds once more
    for g, r in ((k, rk), (v, rv)):
        assert (np.abs(host(g).astype(np.float64) - r) <= np.abs(r) * (2.0 ** -11 + 2.0 ** -23) + 2.0 ** -25).all()
    assert not host(k)[[0, -1]].any() and not host(v)[[0, -1]].any()


@pytest.mark.parametrize("page,dim,layout,rot,given", [(64, 128, "half", 128, False), (16, 64, "pairs", 32, True),
                                                       (32, 80, "half", 20, False), (128, 256, "half", 256, True)])
def test_append_rotates(page, dim, layout, rot, given):
    rng = np.random.default_rng(dim)
    heads, Hq, news, lens = 2, 6, [70, 1, 0, 9], [75, 300, 4, 9]
    T = sum(news) + 4
    pages = sum(-(-L // page) for L in lens) + 1
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng, lead=1)
    want = filled_cache(pages, heads, dim, page, rng)
    cache = to_device(want)
    before = want.copy()
    K, V, q = normal(rng, T, heads, dim), normal(rng, T, heads, dim), normal(rng, T, Hq, dim)
    freq = A.frequencies(rot, 1e4)
    pos = rng.integers(0, 100000, T).astype(np.int32) if given else None
    p = pos if given else A.positions(cu, ln, T)
    q_out = strided(np.full_like(q, 5))
    r = sq.kv_append(cache, strided(K), strided(V), dev(cu), dev(ln), dev(table), freq=dev(freq), pos=dev(pos),
                     layout=layout, amplitude=1.1, q=strided(q), q_out=q_out)
    assert r is q_out
    # queries: exactly the rotation alone; rows of no sequence as they were
    rows = np.r_[cu[0]:cu[-1]]
    alone = host(sq.rope(dev(q), dev(freq), dev(p.astype(np.int32)), layout=layout, amplitude=1.1))
    assert_bits(host(q_out)[rows], alone[rows], "q")
    rest = np.setdiff1d(np.arange(T), rows)
    assert (host(q_out)[rest] == 5).all()
    # values bit-exact, keys within the bound of the exact rotation
    Kr = A.rope(K, p, freq, layout, 1.1)
    A.append(want, Kr, V.astype(np.float32), cu, ln, table)
    assert_bits(host(cache.v), want.v, "v")
    assert_bits(host(cache.v_scale), want.vs, "v_scale")
    ks, k = host(cache.k_scale).astype(np.float64), host(cache.k)
    assert (np.abs(ks / want.ks - 1) <= 2.0 ** -20).all()
    written = np.zeros(want.k.shape[:3], bool)
    for pid, s0, s1, t in A.spans(cu, ln, table, page, pages):
        for h in range(heads):
            x = Kr[t:t + s1 - s0, h] / ks[pid, h]
            assert (np.abs(k[pid, h, s0:s1] - x) <= 0.5 + 127 * 2.0 ** -19).all()
            if s0:                                                # older codes, rescaled where the scale grew
                o = before.k[pid, h, :s0] * (before.ks[pid, h] / ks[pid, h])
                assert (np.abs(k[pid, h, :s0] - o) <= 0.5 + 127 * 2.0 ** -19).all()
            written[pid, h, :s1] = True
    assert np.array_equal(k[~written], before.k[~written])


def test_zero_and_extreme_rows():
    """Zero rows (scale 0, codes 0), the largest and smallest fp16, and a scale that does not shrink."""
    rng = np.random.default_rng(2)
    K = np.zeros((5, 1, 16), np.float16)
    K[1] = 65504
    K[2] = 6e-8
    K[3, 0, 3] = -65504
    V = K[::-1].copy()
    want = A.Cache(5, 1, 16, 16)
    cache = to_device(want)
    cu, ln, table = ragged([1] * 5, [1] * 5, 1, 16, 5, rng)
    sq.kv_append(cache, dev(K), dev(V), dev(cu), dev(ln), dev(table))
    A.append(want, K.astype(np.float32), V.astype(np.float32), cu, ln, table)
    same_cache(cache, want, "one token each")
    for L in (2, 3, 4):                                           # a page filled token by token
        K = normal(rng, 5, 1, 16, scale=10.0 ** (3 - L))
        ln = np.full(5, L, np.int32)
        sq.kv_append(cache, dev(K), dev(K), dev(cu), dev(ln), dev(table))
        A.append(want, K.astype(np.float32), K.astype(np.float32), cu, ln, table)
        same_cache(cache, want, f"length {L}")


def test_bad_index_values_write_nothing_outside():
    """Lengths, rows and pages out of range: clamped or dropped, every other page as it was."""
    rng = np.random.default_rng(3)
    want = filled_cache(6, 2, 32, 16, rng)
    K = normal(rng, 8, 2, 32)
    for cu, ln, table in (([0, 4, 8], [4, 4], [[-1, 2], [6, 3]]),               # no such pages
                          ([0, 4, 8], [-5, 4], [[0, 1], [2 ** 31 - 1, 3]]),     # a negative length
                          ([-3, 0, 0], [10, 10], [[0, 1], [2, 3]]),             # rows before the first: none
                          ([8, 20, 90], [12, 5], [[0, 1], [2, 3]]),             # rows past the last: none
                          ([6, 2, 1], [2, 2], [[0, 1], [2, 3]])):               # decreasing: none
        cache = to_device(want)
        cu, ln, table = np.array(cu, np.int32), np.array(ln, np.int32), np.array(table, np.int32)
        sq.kv_append(cache, dev(K), dev(K), dev(cu), dev(ln), dev(table))
        out = sq.attn_kv8(dev(K), cache, dev(cu), dev(ln), dev(table))
        torch.cuda.synchronize()
        same_cache(cache, want, str(cu))
        assert out.shape == K.shape


def test_length_past_the_table_is_clamped():
    rng = np.random.default_rng(4)
    want = filled_cache(4, 1, 16, 16, rng)
    cache = to_device(want)
    K = normal(rng, 3, 1, 16)
    table = np.array([[2, 0]], np.int32)
    sq.kv_append(cache, dev(K), dev(K), dev(np.array([0, 3], np.int32)), dev(np.array([1000], np.int32)), dev(table))
    A.append(want, K.astype(np.float32), K.astype(np.float32), np.array([0, 3]), np.array([32]), table)
    same_cache(cache, want, "clamped")


def test_large_offsets():
    """Pages past 2^31 bytes of codes."""
    pages, heads, dim, page = 2 ** 31 // (8 * 128 * 128) + 40, 8, 128, 128
    c = sq.kv_cache(pages, heads, dim, page)
    rng = np.random.default_rng(5)
    K = normal(rng, 1, heads, dim)
    cu, ln = np.array([0, 1], np.int32), np.array([1], np.int32)
    last = pages - 1
    sq.kv_append(c, dev(K), dev(K), dev(cu), dev(ln), dev(np.array([[last]], np.int32)))
    k, v = sq.kv_read(c, dev(np.array([last, 0], np.int32)))
    s = np.abs(K.astype(np.float64)).max(-1)[0] / 127
    for x in (host(k), host(v)):
        assert (np.abs(x[0, :, 0].astype(np.float64) - K[0]) <= s[:, None] * 0.51 + 2.0 ** -10).all()
        assert not x[1].any() and not x[0, :, 1:].any()
    out = host(sq.attn_kv8(dev(K), c, dev(cu), dev(ln), dev(np.array([[last]], np.int32))))
    assert (np.abs(out[0].astype(np.float64) - K[0]) <= s[:, None] * 0.51 + 2.0 ** -9).all()
