"""Rotary positions, the 8-bit cache, attention and weight-only products at the ends of
what their interface allows: offsets past 32 bits, the most sequences, pages shared by
sequences, queries that are not finite, rows that touch the end of a buffer."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, normal, ragged, to_device
from gpu_util import assert_bits, dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu

FAR = 2 ** 28                          # elements between rows: the ninth row begins at 2^31


def far(a):
    """a [9, H, D] on the device with its rows FAR elements apart."""
    T, H, D = a.shape
    x = torch.empty((T - 1) * FAR + H * D, dtype=torch.float16, device="cuda").as_strided((T, H, D), (FAR, D, 1))
    x.copy_(dev(a))
    return x


def test_strides_past_32_bits():
    rng = np.random.default_rng(1)
    heads, G, dim, page = 2, 3, 64, 16
    K, V, q = normal(rng, 9, heads, dim), normal(rng, 9, heads, dim), normal(rng, 9, heads * G, dim)
    freq = dev(A.frequencies(dim, 1e4))
    cu, ln, table = ragged([4, 5], [30, 5], 2, page, 8, rng)
    args = (dev(cu), dev(ln), dev(table))
    near = to_device(filled_cache(8, heads, dim, page, np.random.default_rng(2)))
    q_near = sq.kv_append(near, dev(K), dev(V), *args, freq=freq, q=dev(q))
    out = host(sq.attn_kv8(q_near, near, *args))
    fq = far(q)
    assert_bits(host(sq.rope(fq, freq)), host(sq.rope(dev(q), freq)), "rope")
    away = to_device(filled_cache(8, heads, dim, page, np.random.default_rng(2)))
    r = sq.kv_append(away, far(K), far(V), *args, freq=freq, q=fq, q_out=fq)
    assert r is fq
    for a, b in zip(away, near):
        assert_bits(host(a), host(b), "cache")
    assert_bits(host(fq.contiguous()), host(q_near), "queries")
    assert_bits(host(sq.attn_kv8(fq, away, *args)), out, "attention")


@pytest.mark.parametrize("news", [3, 12])          # tiles of 128 rows, by the many rows before them
def test_outputs_past_32_bits(news):
    """Rows behind 70000 others, which see nothing: their outputs begin past 2^31 elements."""
    heads, G, dim, page, T = 8, 16, 256, 64, 70000
    rng = np.random.default_rng(news)
    c = filled_cache(6, heads, dim, page, rng)
    cu, ln = np.array([0, T - news, T], np.int32), np.array([0, 200], np.int32)
    table = np.array([[-1] * 4, [3, 5, 0, 1]], np.int32)
    q = torch.zeros(T, heads * G, dim, dtype=torch.float16, device="cuda")
    tail = normal(rng, news, heads * G, dim)
    q[T - news:] = dev(tail)
    out, lse = sq.attn_kv8(q, to_device(c), dev(cu), dev(ln), dev(table), want_lse=True)
    ref = A.attention(tail, c, np.array([0, news], np.int32), ln[1:], table[1:])
    check_attention(out[T - news:].contiguous(), ref, news, lse[T - news:].contiguous())
    assert not out[:T - news].any() and torch.isneginf(lse[:T - news]).all()


def test_rotates_past_32_bits():
    x = torch.zeros(2 ** 16 + 3, 512, 64, dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(3)
    tail = normal(rng, 3, 512, 64)
    x[-3:] = dev(tail)
    freq = dev(A.frequencies(64, 1e4))
    pos = torch.arange(2 ** 16 + 3, dtype=torch.int32, device="cuda") - 2 ** 16
    want = host(sq.rope(dev(tail), freq, dev(np.array([0, 1, 2], np.int32))))
    sq.rope(x, freq, pos, out=x)
    assert_bits(host(x[-3:].contiguous()), want, "tail")
    assert not x[:-3].any()
    y = x[:, :, :32].unflatten(2, (1, 2, 16))[:, :, 0, 0]      # a view: heads of 16 inside rows of 64
    part = host(sq.rope(y[-3:], dev(A.frequencies(6, 1e4))))
    assert_bits(part[:, :, 6:], want[:, :, 6:16], "behind the rotated part")


def test_most_sequences():
    """2^14 sequences of a token each, appended and read."""
    B, heads, dim, page = 2 ** 14, 1, 16, 16
    rng = np.random.default_rng(4)
    want = A.Cache(B, heads, dim, page)
    cache = to_device(want)
    table = rng.permutation(B).astype(np.int32)[:, None]
    cu = np.arange(B + 1, dtype=np.int32)
    for L in (1, 2):
        K, V, q = normal(rng, B, heads, dim), normal(rng, B, heads, dim), normal(rng, B, 2, dim)
        ln = np.full(B, L, np.int32)
        ln[rng.integers(0, B, 50)] = 0
        sq.kv_append(cache, dev(K), dev(V), dev(cu), dev(ln), dev(table))
        A.append(want, K.astype(np.float32), V.astype(np.float32), cu, ln, table)
        for a, b in zip(cache, (want.k, want.v, want.ks, want.vs)):
            assert_bits(host(a), b, f"length {L}")
        out, lse = sq.attn_kv8(dev(q), cache, dev(cu), dev(ln), dev(table), want_lse=True)
        check_attention(out, A.attention(q, want, cu, ln, table), L, lse)
    with pytest.raises(sq.StarQuantError, match="B="):
        sq.attn_kv8(dev(q), cache, dev(np.arange(B + 2, dtype=np.int32)), dev(np.zeros(B + 1, np.int32)),
                    torch.zeros(B + 1, 1, dtype=torch.int32, device="cuda"))


def test_heads_that_do_not_divide_the_workgroups():
    """Three key heads over a grid of a fixed number of workgroups, nearly all of them with a tile."""
    page, heads, G, dim, n, B = 64, 3, 2, 16, 1490, 7
    rng = np.random.default_rng(7)
    pages = B * 24
    cu, ln, table = ragged([n] * B, [n] * B, 24, page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    q = normal(rng, n * B, heads * G, dim)
    out = torch.full((n * B, heads * G, dim), 9.0, dtype=torch.float16, device="cuda")
    sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), causal=False, out=out)
    rows = np.r_[0:3, 700:703, cu[1:] - 1, cu[1:-1], n * B - 130:n * B]
    got = host(out)
    assert not (got == 9).all(-1).any()
    for b in range(B):
        t = rows[(rows >= cu[b]) & (rows < cu[b + 1])]
        one = np.array([0, len(t)], np.int32)
        ref = A.attention(q[t], c, one, ln[b:b + 1], table[b:b + 1], causal=False)
        check_attention(got[t], ref, b)


@pytest.mark.parametrize("news", [[1, 1, 1], [20, 9, 1], [70, 100, 90]])
def test_sequences_share_pages(news):
    """A common beginning in the same pages, several times the same page in one sequence; pages read back twice."""
    page, heads, G, dim = 16, 2, 4, 64
    rng = np.random.default_rng(5)
    c = filled_cache(30, heads, dim, page, rng)
    lens = [150, 140, 100]
    table = np.full((3, 10), -1, np.int32)
    table[:, :5] = [7, 2, 2, 9, 4]
    table[:, 5:] = rng.permutation(np.setdiff1d(np.arange(30), [7, 2, 9, 4]))[:15].reshape(3, 5)
    cu, ln = np.r_[0, np.cumsum(news)].astype(np.int32), np.array(lens, np.int32)
    q = normal(rng, sum(news), heads * G, dim)
    out, lse = sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), want_lse=True)
    check_attention(out, A.attention(q, c, cu, ln, table), news, lse)
    k, v = sq.kv_read(to_device(c), dev(np.array([2, 7, 2], np.int32)))
    assert_bits(host(k[0]), host(k[2]), "k")
    assert_bits(host(v[0]), host(v[2]), "v")


@pytest.mark.parametrize("news,lens", [([3, 2], [90, 70]), ([20, 12], [90, 70]), ([90, 60], [90, 70]),
                                       ([2, 1], [5000, 70]), ([70, 100], [3000, 100])])
def test_queries_that_are_not_finite(news, lens):
    """NaN and infinite queries spoil their own rows alone."""
    page, heads, G, dim = 64, 2, 4, 64
    rng = np.random.default_rng(6)
    pages = sum(-(-L // page) for L in lens)
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    q = normal(rng, sum(news), heads * G, dim)
    bad = q.copy()
    rows = [(0, 1), (sum(news) - 1, heads * G - 1)]
    bad[rows[0]] = np.nan
    bad[rows[1]][::2] = np.inf
    out, lse = (host(t) for t in sq.attn_kv8(dev(bad), to_device(c), dev(cu), dev(ln), dev(table), want_lse=True))
    ref = A.attention(q, c, cu, ln, table)
    for t, h in rows:
        assert np.isnan(out[t, h]).all() and np.isnan(lse[t, h])
        out[t, h], lse[t, h] = ref[0][t, h], ref[1][t, h]
    check_attention(dev(out), ref, news, dev(lse))


def test_binding_refuses_workspaces_and_outputs():
    rng = np.random.default_rng(8)
    c = filled_cache(40, 2, 64, 64, rng)
    cu, ln, table = ragged([1], [2000], 32, 64, 40, rng)
    q = dev(normal(rng, 1, 8, 64))
    args = (to_device(c), dev(cu), dev(ln), dev(table))
    need = sq.attn_kv8_workspace_bytes(1, 1, 8, 2, 64, 32 * 64)
    for kw, what in ((dict(ws=torch.empty(need, dtype=torch.uint8)), "ws"),
                     (dict(ws=torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]), "ws"),
                     (dict(out=torch.empty(1, 8, 64, dtype=torch.float16)), "out"),
                     (dict(lse=torch.empty(1, 7, dtype=torch.float32, device="cuda")), "lse")):
        with pytest.raises(ValueError, match=what):
            sq.attn_kv8(q, *args, **kw)
    with pytest.raises(sq.StarQuantError, match="overlap"):
        sq.attn_kv8(q, *args, out=q)


@pytest.mark.parametrize("M", [1, 2, 17, 33, 65, 4099])
@pytest.mark.parametrize("K,group", [(64, 32), (192, 64), (1088, 32)])
def test_weight_only_rows_stay_apart(M, K, group):
    """K of half a step: what lies behind a row's end, a row of infinities or nothing, does not enter."""
    rng = np.random.default_rng(M + K)
    W = normal(rng, 40, K, scale=0.05)
    Wq, s = sq.quantize_weights_group(dev(W), group)
    Wf = sq.weights_to_frag(Wq)
    X = normal(rng, M, K)
    want = host(sq.w4a16_gemm_frag(dev(X), Wf, s))
    assert np.isfinite(want).all()
    X[1::2] = np.inf
    got = host(sq.w4a16_gemm_frag(dev(X), Wf, s))
    assert_bits(got[::2], want[::2], "finite rows")
    assert not np.isfinite(got[1::2]).any()
