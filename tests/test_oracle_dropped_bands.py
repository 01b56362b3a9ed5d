"""The oracle's codes of rows that are not finite where their state drops them."""
import numpy as np

from oracle import layer as L


def test_a_row_that_holds_an_infinity_has_no_scale():
    h = np.ones((4, 64), np.float16)
    h[1, 63] = h[2, 61] = h[3, 63] = np.inf            # dropped by masked, unmasked and masked rows
    state = np.array([0, 1, 0, 0], np.uint8)
    n, _ = L.norm(h)
    assert (n[1, :63] == 0).all() and np.isnan(n[1, 63])
    q, s = L.quantise_gated(n, state, 2, 2, 4)
    assert np.isfinite(s[0]) and np.isnan(s[1:]).all() and (q[1:] == 0).all() and (q[0] != 0).any()


def test_finite_rows_are_the_gated_rows():
    n = np.random.default_rng(1).normal(0, 1, (6, 128)).astype(np.float32)
    state = np.array([0, 1, 1, 0, 2, 0], np.uint8)
    for bits in (4, 8):
        for a, b in zip(L.quantise_gated(n, state, 9, 5, bits), L.quantise(L.gated(n, state, 9, 5), bits)):
            assert a.tobytes() == b.tobytes()
