"""Every page and head size of the cache, bit-exact against the oracle: whole and partial
pages, older codes rescaled, pages read back; and rotated parts of every remainder."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import filled_cache, normal, ragged, to_device
from gpu_util import assert_bits, dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", list(range(16, 257, 16)))
def test_append_and_read(page, dim):
    rng = np.random.default_rng(page + dim)
    heads, news, lens = 2, [page + 7, 1, 3], [2 * page, page + 2, page]
    pages = sum(-(-L // page) for L in lens) + 1
    cu, ln, table = ragged(news, lens, 2, page, pages, rng)
    want = filled_cache(pages, heads, dim, page, rng)
    cache = to_device(want)
    K, V = normal(rng, sum(news), heads, dim, scale=2), normal(rng, sum(news), heads, dim)
    V[::2] *= np.float16(5)
    sq.kv_append(cache, dev(K), dev(V), dev(cu), dev(ln), dev(table))
    A.append(want, K.astype(np.float32), V.astype(np.float32), cu, ln, table)
    for name, x, y in zip(("k", "v", "k_scale", "v_scale"), cache, (want.k, want.v, want.ks, want.vs)):
        assert_bits(host(x), y, name)
    pids = np.arange(pages, dtype=np.int32)
    # code times scale in fp32, one rounding to fp16
    for g, r in zip(sq.kv_read(cache, dev(pids)), A.values(want, pids)):
        assert (np.abs(host(g).astype(np.float64) - r) <= np.abs(r) * (2.0 ** -11 + 2.0 ** -23) + 2.0 ** -25).all()


@pytest.mark.parametrize("page,dim,rot", [(128, 256, 250), (128, 256, 2), (16, 16, 14), (64, 128, 126), (32, 96, 24),
                                          (128, 80, 40), (64, 256, 256), (128, 128, 96)])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotated_parts(page, dim, rot, layout):
    """Keys against the rotation alone, whose fp16 results are within 2^-11 and its own arithmetic of the keys that
    are quantised; values bit-exact."""
    rng = np.random.default_rng(rot)
    heads, news, lens = 2, [page + 3], [2 * page - 1]
    cu, ln, table = ragged(news, lens, 2, page, 3, rng)
    want = A.Cache(3, heads, dim, page)
    cache = to_device(want)
    K, V, q = normal(rng, news[0], heads, dim), normal(rng, news[0], heads, dim), normal(rng, news[0], 3, dim)
    freq = A.frequencies(rot, 1e4)
    p = A.positions(cu, ln, news[0])
    qr = sq.kv_append(cache, dev(K), dev(V), dev(cu), dev(ln), dev(table), freq=dev(freq), layout=layout, q=dev(q))
    assert_bits(host(qr), host(sq.rope(dev(q), dev(freq), dev(p.astype(np.int32)), layout=layout)), "q")
    Kr = A.rope(K, p, freq, layout)
    A.append(want, Kr, V.astype(np.float32), cu, ln, table)
    assert_bits(host(cache.v), want.v, "v")
    ks, k = host(cache.k_scale).astype(np.float64), host(cache.k)
    for pid, s0, s1, t in A.spans(cu, ln, table, page, 3):
        for h in range(heads):
            assert abs(ks[pid, h] / want.ks[pid, h] - 1) <= 2.0 ** -20
            x = Kr[t:t + s1 - s0, h] / ks[pid, h]
            assert (np.abs(k[pid, h, s0:s1] - x) <= 0.5 + 127 * 2.0 ** -19).all()
