"""Sizes whose grid would have 2^32 threads, which no launch takes, are turned down with the
others that are too large; those just below are not (their missing pointers are found next).
Workgroups are of 256 threads, so 2^24 of them are one too many."""
import pytest

from paper_2606_04945_amd import _lib as L

FAKE = 1 << 20          # a 16-byte aligned non-null address; never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    return L.lib()


@pytest.mark.parametrize("D", [16, 48])
def test_rope(lib, D):
    """One head: T D / 2 threads where rot % 16 != 0, an eighth of that elsewhere."""
    def rope(T, rot):
        return lib.sq_rope(None, D, D, None, FAKE, T, 1, D, rot, 0, 0, 1.0, None, D, D, None)
    most, odd = (2 ** 33 - 1) // D, (2 ** 33 - 512) // D
    assert odd < most
    assert rope(most, 16) == L.SQ_ERR_NULL and rope(most + 1, 16) == L.SQ_ERR_SHAPE
    assert rope(odd, 6) == L.SQ_ERR_NULL and rope(odd + 1, 6) == L.SQ_ERR_SHAPE and rope(most, 6) == L.SQ_ERR_SHAPE


@pytest.mark.parametrize("dim,page,heads,T", [(16, 16, 16, 16268784), (80, 16, 18, 13094384), (96, 32, 30, 14913041)])
def test_append(lib, dim, page, heads, T):
    """Pages take 2^24 - 1 workgroups together with the full ones of one query head; one more is not full."""
    assert (T // page + 2) * heads + T * dim // 512 == 2 ** 24 - 1 and T * dim % 512

    def append(T):
        c = L.KVCacheStruct(FAKE, FAKE, FAKE, FAKE, 4, page, heads, dim)
        s = (heads * dim, dim)
        return lib.kv_append(c, None, *s, FAKE, *s, FAKE, FAKE, FAKE, T, 1, 4, None, FAKE, 2, 0, 1.0, FAKE, dim, dim, 1,
                             FAKE << 1, dim, dim, None)
    assert append(T) == L.SQ_ERR_SHAPE
    assert append(T - page) == L.SQ_ERR_NULL


def test_quantize_group(lib):
    """A wave a group, four a workgroup: rows come in eights, so the largest number of groups is 2^26 - 8."""
    f = lib.sq_quantize_weights_group
    assert f(None, 2 ** 25, 64, 32, None, None, None) == L.SQ_ERR_SHAPE
    assert f(None, 2 ** 25 - 8, 64, 32, None, None, None) == L.SQ_ERR_NULL
