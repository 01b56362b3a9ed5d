"""Pins of the oracle for rotary positions, the 8-bit cache, attention and weight-only
products: values worked out by hand or by another formula."""
import numpy as np

from oracle import attn as A


def test_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    x, pos, f = rng.standard_normal((4, 2, 8)), np.array([0, 3, 10, -2]), A.frequencies(8, 100.0)
    for layout in ("half", "pairs"):
        a, b = A.pair_index(8, layout)
        z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None, None] * f)
        y = A.rope(x, pos, f, layout, 1.5)
        assert np.allclose(y[..., a], z.real, atol=1e-14) and np.allclose(y[..., b], z.imag, atol=1e-14)
        assert np.allclose(A.rope(A.rope(x, pos, f, layout), pos, f, layout, transpose=True), x, atol=1e-14)
    quarter = A.rope(np.array([[[1.0, 2.0, 9.0]]])[..., :2], np.array([1]), np.array([np.pi / 2]))
    assert np.allclose(quarter, [[[-2, 1]]], atol=1e-15)


def test_frequencies_by_hand():
    assert np.allclose(A.frequencies(4, 100.0), [1, 0.1])
    assert np.allclose(A.frequencies(4, 100.0, "linear", 4.0), [0.25, 0.025])
    assert np.allclose(A.frequencies(4, 100.0, "ntk", 4.0), [1, 0.1 / 4])             # the last pair: all of the factor
    f = A.frequencies(4, 100.0, "yarn", 4.0, original=2 * np.pi * 16.5, beta_fast=32, beta_slow=1)
    assert np.allclose(f, [0.5 + 0.5 / 4, (0.65 / 31) * 0.1 + (1 - 0.65 / 31) * 0.025])   # 16.5 and 1.65 turns


def test_append_by_hand():
    c = A.Cache(2, 1, 1, 16)
    table = np.array([[1]])
    one = lambda v: np.array([[[v]]], np.float32)  # noqa: E731
    A.append(c, one(127.0), one(-12.7), [0, 1], [1], table)
    assert c.ks[1, 0] == 1 and c.k[1, 0, 0, 0] == 127 and c.v[1, 0, 0, 0] == -127 and not c.k[0].any()
    A.append(c, one(64.0), one(0.0), [0, 1], [2], table)                  # smaller: the scale stays
    assert c.ks[1, 0] == 1 and c.k[1, 0, 1, 0] == 64
    A.append(c, one(-254.0), one(0.0), [0, 1], [3], table)                # larger: older codes halve, ties to even
    assert c.ks[1, 0] == 2 and c.k[1, 0, :3, 0].tolist() == [64, 32, -127]
    before = c.copy()
    A.append(c, one(-254.0), one(0.0), [0, 1], [3], table)
    assert np.array_equal(c.k, before.k)
    A.append(c, one(3.0), one(0.0), [0, 1], [1], table)                   # slot 0 again: a scale of its own
    assert c.ks[1, 0] == np.float32(3) / np.float32(127) and c.k[1, 0, 0, 0] == 127


def test_spans():
    t = np.array([[4, 5, 6], [7, 8, -1]])
    assert A.spans([0, 20, 23], [40, 33], t, 16, 9) == [(5, 4, 16, 0), (6, 0, 8, 12), (8, 14, 16, 20)]
    assert A.spans([0, 5], [3], t, 16, 9) == [(4, 0, 3, 2)]               # two tokens before position 0


def test_attention_against_a_matrix_form():
    rng = np.random.default_rng(1)
    c = A.Cache(5, 2, 8, 16)
    c.k = rng.integers(-127, 128, c.k.shape).astype(np.int8)
    c.v = rng.integers(-127, 128, c.v.shape).astype(np.int8)
    c.ks[:], c.vs[:] = 0.01, rng.uniform(0.01, 0.02, c.vs.shape)
    table = np.array([[3, 0, 4]])
    q = rng.standard_normal((4, 6, 8))
    for causal, window in ((False, 0), (True, 0), (True, 5)):
        out, lse, _ = A.attention(q, c, [0, 4], [39], table, causal, window)
        k, v = A.values(c, table[0])
        k, v = (x.transpose(1, 0, 2, 3).reshape(2, 48, 8).repeat(3, 0) for x in (k, v))
        s = np.einsum("thd,hkd->htk", q, k) / 8 ** 0.5
        p, j = np.arange(35, 39)[:, None], np.arange(48)
        mask = (j >= 39) | (causal & (j > p)) | ((window > 0) & (j <= p - window))
        s = np.where(mask[None], -np.inf, s)
        w = np.exp(s) / np.exp(s).sum(-1, keepdims=True)
        assert np.allclose(out, np.einsum("htk,hkd->thd", w, v), atol=1e-12)
        assert np.allclose(lse, np.log(np.exp(s).sum(-1)).T, atol=1e-12)
    out, lse, _ = A.attention(q, c, [0, 4], [2], table)                   # the first two queries see nothing
    assert not out[:2].any() and np.isneginf(lse[:2]).all() and out[2:].all()


def test_group_quantiser_by_hand():
    W = np.array([[7, -7, 3.5, 0.5] + [0] * 28 + [-14, 2] + [0] * 30], np.float16)
    q, s = A.quantize_group(W, 32)
    assert s[:, 0].tolist() == [1, 2] and q[0, :4].tolist() == [7, -7, 4, 0] and q[0, 32:34].tolist() == [-7, 1]
    y, mass = A.w4a16(np.ones((1, 64), np.float16), q, s, 32)
    assert y[0, 0] == 4 - 12 and mass[0, 0] == 18 + 16
