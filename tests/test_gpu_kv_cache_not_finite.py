"""Keys and values that are not finite: their page's scale says so, and reading the page or
attending to it gives NaN, until its slot 0 is written again."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import filled_cache, normal, ragged, strided, to_device
from gpu_util import assert_bits, dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


def same(cache, want, what):
    for name, x, y in zip(("k", "v"), cache, (want.k, want.v)):
        assert_bits(host(x), y, f"{what}: {name}")
    for x, y in ((cache.k_scale, want.ks), (cache.v_scale, want.vs)):
        assert np.array_equal(host(x), y, equal_nan=True), what


@pytest.mark.parametrize("page,heads,dim,news,lens", [(16, 2, 16, [3], [8]), (64, 2, 128, [130, 1], [140, 70]),
                                                      (32, 3, 80, [33, 1], [64, 33]), (128, 1, 256, [129, 5], [140, 127])])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_scales_tell(page, heads, dim, news, lens, value):
    rng = np.random.default_rng(page + dim)
    T = sum(news)
    pages = sum(-(-L // page) for L in lens) + 1
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    want = filled_cache(pages, heads, dim, page, rng)
    cache = to_device(want)
    K, V = normal(rng, T, heads, dim), normal(rng, T, heads, dim)
    K[0, 0, dim - 1] = value
    V[T - 1, heads - 1, 3] = value
    args = (strided(K), strided(V), dev(cu), dev(ln), dev(table))
    sq.kv_append(cache, *args)
    A.append(want, K.astype(np.float32), V.astype(np.float32), cu, ln, table)
    assert (~np.isfinite(want.ks)).sum() == 1 and (~np.isfinite(want.vs)).sum() == 1
    same(cache, want, "first")
    sq.kv_append(cache, *args)
    same(cache, want, "again")
    pk, pv = int(np.argwhere(~np.isfinite(want.ks))[0, 0]), int(np.argwhere(~np.isfinite(want.vs))[0, 0])
    k, v = (host(t) for t in sq.kv_read(cache, dev(np.array([pk, pv], np.int32))))
    assert np.isnan(k[0, 0]).all() and np.isnan(v[1, -1]).all()
    assert np.isfinite(k[0, 1:]).all() and np.isfinite(v[1, :-1]).all()
    out = host(sq.attn_kv8(dev(normal(rng, T, heads, dim)), cache, dev(cu), dev(ln), dev(table)))
    assert np.isnan(out[0, 0]).all() and np.isnan(out[T - 1, -1]).all()
    # finite tokens behind them do not hide it
    cu1, t1 = np.array([0, 1], np.int32), np.array([[pk]], np.int32)
    last = np.array([page], np.int32)
    x = normal(rng, 1, heads, dim)
    sq.kv_append(cache, dev(x), dev(x), dev(cu1), dev(last), dev(t1))
    A.append(want, x.astype(np.float32), x.astype(np.float32), cu1, last, t1)
    assert not np.isfinite(want.ks[pk, 0])
    same(cache, want, "a finite token")
    # the page taken anew
    last[0] = 1
    sq.kv_append(cache, dev(x), dev(x), dev(cu1), dev(last), dev(t1))
    A.append(want, x.astype(np.float32), x.astype(np.float32), cu1, last, t1)
    assert np.isfinite(want.ks[pk]).all()
    same(cache, want, "anew")


@pytest.mark.parametrize("rot", [64, 20])
def test_rotated_keys_that_pass_fp32(rot):
    """A finite key that its rotation's amplitude takes out of fp32."""
    rng = np.random.default_rng(rot)
    page, heads, dim = 32, 2, 64
    want = filled_cache(3, heads, dim, page, rng)
    cache = to_device(want)
    K = normal(rng, 2, heads, dim)
    K[1, 1, 2] = 60000
    cu, ln, table = np.array([0, 2], np.int32), np.array([9], np.int32), np.array([[1]], np.int32)
    sq.kv_append(cache, dev(K), dev(K), dev(cu), dev(ln), dev(table), freq=dev(A.frequencies(rot, 1e4)), amplitude=1e34)
    ks = host(cache.k_scale)
    assert not np.isfinite(ks[1, 1]) and np.isfinite(ks[1, 0]) and np.isfinite(host(cache.v_scale)).all()
    k, _ = sq.kv_read(cache, dev(np.array([1], np.int32)))
    assert np.isnan(host(k)[0, 1]).all()
