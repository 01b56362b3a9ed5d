"""Host-side refusals of the rotary, cache, attention and weight-only entry points:
every bad argument is turned down before anything touches a device."""
import ctypes

import pytest
import torch

import paper_2606_04945_amd as sq
from paper_2606_04945_amd import _lib as L

FAKE = 1 << 20          # a 16-byte aligned non-null address; never dereferenced on these paths
BAD = FAKE + 2
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return L.lib()


def cache(**kw):
    f = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, pages=4, page=64, heads=2, dim=64)
    f.update(kw)
    return L.KVCacheStruct(*(f[n] for n, _ in L.KVCacheStruct._fields_))


def rope(lib, **kw):
    a = dict(X=FAKE, xt=128, xh=64, pos=None, freq=FAKE, T=4, H=2, D=64, rot=64, layout=0, tr=0, amp=1.0, Y=FAKE << 1,
             yt=128, yh=64)
    a.update(kw)
    return lib.sq_rope(*a.values(), None)


def test_rope(lib):
    for kw in (dict(D=24), dict(D=0), dict(D=1040, rot=64, xt=2080, yt=2080, yh=1040), dict(rot=0), dict(rot=3),
               dict(rot=66), dict(layout=2), dict(layout=-1), dict(amp=NAN), dict(amp=INF), dict(T=-1), dict(H=-1),
               dict(xt=129), dict(xh=-64), dict(yt=64), dict(yh=32), dict(yt=8, yh=64),
               dict(T=1 << 24, H=1024, D=64), dict(T=1 << 20, H=128, D=64, xh=64, xt=8192, yt=8192), dict(Y=FAKE, yt=256)):
        assert rope(lib, **kw) == L.SQ_ERR_SHAPE, kw
    for kw in (dict(X=None), dict(Y=None), dict(freq=None)):
        assert rope(lib, **kw) == L.SQ_ERR_NULL, kw
    for kw in (dict(X=BAD), dict(Y=BAD), dict(freq=FAKE + 8), dict(pos=BAD)):
        assert rope(lib, **kw) == L.SQ_ERR_ALIGN, kw
    assert rope(lib, T=0, X=None) == L.SQ_OK and rope(lib, H=0, Y=None) == L.SQ_OK


def test_rope_frequencies(lib):
    f = lib.sq_rope_frequencies
    for a in ((0, 1e4, 0, 1, 0, 32, 1), (7, 1e4, 0, 1, 0, 32, 1), (1026, 1e4, 0, 1, 0, 32, 1), (64, 1.0, 0, 1, 0, 32, 1),
              (64, NAN, 0, 1, 0, 32, 1), (64, INF, 0, 1, 0, 32, 1), (64, 1e4, 4, 1, 0, 32, 1), (64, 1e4, 1, .5, 0, 32, 1),
              (64, 1e4, 2, NAN, 0, 32, 1), (64, 1e4, 3, 2, 0, 32, 1), (64, 1e4, 3, 2, 10, 1, 1),
              (64, 1e4, 3, 2, 10, 2, -1), (64, 1e4, 3, 2, NAN, 32, 1)):
        assert f(*a, FAKE, None) == L.SQ_ERR_SHAPE, a
    assert f(64, 1e4, 0, 1, 0, 32, 1, None, None) == L.SQ_ERR_NULL
    assert f(64, 1e4, 0, 1, 0, 32, 1, BAD, None) == L.SQ_ERR_ALIGN
    assert lib.sq_rope_amplitude(1, 8.0) == 1.0 and abs(lib.sq_rope_amplitude(3, 8.0) - 1.2079441541679836) < 1e-15


CACHE_SHAPE = (dict(page=0), dict(page=48), dict(page=256), dict(dim=0), dict(dim=72), dict(dim=272), dict(heads=0),
               dict(heads=1025), dict(pages=0))
CACHE_NULL = (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None))


def append(lib, c=None, **kw):
    a = dict(K=FAKE, kt=128, kh=64, V=FAKE, vt=128, vh=64, cu=FAKE, lens=FAKE, table=FAKE, T=4, B=2, mp=3, pos=None,
             freq=FAKE, rot=64, layout=0, amp=1.0, Q=FAKE, qt=256, qh=64, Hq=4, R=FAKE << 1, rt=256, rh=64)
    a.update(kw)
    return lib.kv_append(cache(**(c or {})), *a.values(), None)


def test_append(lib):
    for c in CACHE_SHAPE:
        assert append(lib, c) == L.SQ_ERR_SHAPE, c
    for c in CACHE_NULL:
        assert append(lib, c) == L.SQ_ERR_NULL, c
    assert append(lib, dict(v=BAD)) == L.SQ_ERR_ALIGN
    for kw in (dict(T=-1), dict(T=(1 << 24) + 1), dict(B=-1), dict(mp=-1), dict(mp=(1 << 22) + 1), dict(rot=65),
               dict(rot=66), dict(layout=2), dict(amp=NAN), dict(Hq=0), dict(Hq=1025), dict(kt=12), dict(vh=-8),
               dict(qt=4), dict(rt=64), dict(rh=8), dict(R=FAKE, rt=512), dict(B=(1 << 14) + 1),
               dict(T=1 << 24, Hq=1024), dict(B=1 << 14, c=dict(heads=512)), dict(T=1 << 24, Hq=16, rot=2)):
        assert append(lib, **kw) == L.SQ_ERR_SHAPE, kw
    for kw in (dict(K=None), dict(V=None), dict(cu=None), dict(lens=None), dict(table=None), dict(R=None),
               dict(freq=None)):
        assert append(lib, **kw) == L.SQ_ERR_NULL, kw
    for kw in (dict(K=BAD), dict(V=BAD), dict(cu=BAD), dict(lens=BAD), dict(table=BAD), dict(pos=BAD), dict(Q=BAD),
               dict(R=BAD), dict(freq=FAKE + 8)):
        assert append(lib, **kw) == L.SQ_ERR_ALIGN, kw
    assert append(lib, T=0, K=None) == L.SQ_OK and append(lib, B=0, K=None) == L.SQ_OK
    assert lib.kv_append(None, *([None] * 1), 0, 0, None, 0, 0, None, None, None, 0, 0, 0, None, None, 0, 0, 1.0, None, 0,
                         0, 0, None, 0, 0, None) == L.SQ_ERR_NULL


def test_read(lib):
    f = lib.kv_read
    for c in CACHE_SHAPE:
        assert f(cache(**c), FAKE, 2, FAKE, FAKE, None) == L.SQ_ERR_SHAPE, c
    for c in CACHE_NULL:
        assert f(cache(**c), FAKE, 2, FAKE, FAKE, None) == L.SQ_ERR_NULL, c
    assert f(cache(), FAKE, -1, FAKE, FAKE, None) == L.SQ_ERR_SHAPE
    assert f(cache(), FAKE, 1 << 23, FAKE, FAKE, None) == L.SQ_ERR_SHAPE
    assert f(cache(), None, 2, FAKE, FAKE, None) == L.SQ_ERR_NULL
    assert f(cache(), FAKE, 2, None, FAKE, None) == L.SQ_ERR_NULL
    assert f(cache(), FAKE, 2, FAKE, BAD, None) == L.SQ_ERR_ALIGN
    assert f(cache(), BAD, 2, FAKE, FAKE, None) == L.SQ_ERR_ALIGN
    assert f(cache(), None, 0, None, None, None) == L.SQ_OK


def attn(lib, c=None, **kw):
    a = dict(Q=FAKE, qt=256, qh=64, c=cache(**(c or {})), cu=FAKE, lens=FAKE, table=FAKE, T=4, B=2, mp=3, Hq=4, causal=1,
             window=0, scale=0.125, O=FAKE << 1, lse=None, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return lib.attn_kv8(*a.values(), None)


def test_attention(lib):
    for c in CACHE_SHAPE:
        assert attn(lib, c) == L.SQ_ERR_SHAPE, c
    for c in CACHE_NULL:
        assert attn(lib, c) == L.SQ_ERR_NULL, c
    for kw in (dict(T=-1), dict(T=(1 << 24) + 1), dict(B=-1), dict(mp=-1), dict(mp=(1 << 22) + 1), dict(Hq=0),
               dict(Hq=3), dict(Hq=1026), dict(window=-1), dict(scale=NAN), dict(scale=INF), dict(qt=100), dict(qh=-64),
               dict(B=(1 << 14) + 1), dict(T=1 << 24, Hq=32), dict(B=1 << 14, c=dict(heads=512), Hq=512),
               dict(T=1 << 17, B=1 << 14, Hq=512, mp=1 << 22), dict(O=FAKE)):
        assert attn(lib, **kw) == L.SQ_ERR_SHAPE, kw
    for kw in (dict(Q=None), dict(O=None), dict(cu=None), dict(lens=None), dict(table=None)):
        assert attn(lib, **kw) == L.SQ_ERR_NULL, kw
    for kw in (dict(Q=BAD), dict(O=BAD), dict(lse=BAD), dict(ws=BAD), dict(cu=BAD), dict(lens=BAD), dict(table=BAD)):
        assert attn(lib, **kw) == L.SQ_ERR_ALIGN, kw
    assert lib.attn_kv8(FAKE, 256, 64, None, FAKE, FAKE, FAKE, 4, 2, 3, 4, 1, 0, 0.1, FAKE, None, FAKE, 1 << 30,
                        None) == L.SQ_ERR_NULL
    need = lib.sq_attn_kv8_workspace_bytes(4, 2, 4, 2, 64, 640 * 64)
    assert need > 0
    assert attn(lib, mp=640, wsb=need - 1) == L.SQ_ERR_WORKSPACE and attn(lib, mp=640, ws=None) == L.SQ_ERR_WORKSPACE
    assert attn(lib, T=0, Q=None) == L.SQ_OK and attn(lib, B=0, O=None) == L.SQ_OK
    for a in ((0, 1, 4, 2, 64, 192), (1, 0, 4, 2, 64, 192), (1, 1, 3, 2, 64, 192), (1, 1, 4, 0, 64, 192),
              (1, 1, 4, 2, 64, -1), (1, 1, 0, 2, 64, 100)):
        assert lib.sq_attn_kv8_workspace_bytes(*a) == 0, a


def test_weight_only(lib):
    q, g = lib.sq_quantize_weights_group, lib.w4a16_gemm_frag
    for N, K, group in ((8, 100, 32), (8, 128, 16), (8, 128, 96), (8, 192, 128), (12, 128, 32), (-8, 128, 32),
                        (8, 128, 0), (8, 128, -128), (8, 64, 128)):
        assert q(FAKE, N, K, group, FAKE, FAKE, None) == L.SQ_ERR_SHAPE, (N, K, group)
        assert g(FAKE, FAKE, FAKE, 4, N, K, group, FAKE, None) == L.SQ_ERR_SHAPE, (N, K, group)
    assert q(None, 8, 128, 32, FAKE, FAKE, None) == L.SQ_ERR_NULL
    assert q(FAKE, 8, 128, 32, BAD, FAKE, None) == L.SQ_ERR_ALIGN
    assert q(None, 0, 128, 32, None, None, None) == L.SQ_OK
    assert g(FAKE, FAKE, FAKE, -1, 8, 128, 32, FAKE, None) == L.SQ_ERR_SHAPE
    assert g(FAKE, FAKE, FAKE, 1 << 21, 8, 128, 32, FAKE, None) == L.SQ_ERR_SHAPE
    assert g(FAKE, FAKE, FAKE, 1, 1 << 20, 8192, 32, FAKE, None) == L.SQ_ERR_SHAPE      # 4 GiB of codes
    assert g(FAKE, FAKE, FAKE, 1, 8, 128, 32, FAKE, None) == L.SQ_ERR_SHAPE              # Y on X
    assert g(FAKE, None, FAKE, 1, 8, 128, 32, FAKE, None) == L.SQ_ERR_NULL
    assert g(FAKE, FAKE, FAKE + 8, 1, 8, 128, 32, FAKE, None) == L.SQ_ERR_ALIGN
    assert g(None, None, None, 0, 8, 128, 32, None, None) == L.SQ_OK


def test_binding_refuses_host_tensors_and_bad_names():
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    freq = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="device tensor"):
        sq.rope(x, freq)
    with pytest.raises(ValueError, match="scaling"):
        sq.rope_frequencies(64, 1e4, scaling="cubic", out=freq)
    with pytest.raises(ValueError, match="device tensor"):
        sq.kv_cache(2, 2, 64, device="cpu").struct()
    with pytest.raises(ValueError, match="device tensor"):
        sq.quantize_weights_group(torch.zeros(8, 100, dtype=torch.float16), 64)
    with pytest.raises(ValueError, match="scaling"):
        sq.rope_amplitude("half", 2.0)
