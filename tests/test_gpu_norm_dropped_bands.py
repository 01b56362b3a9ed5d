"""Entries that are not finite in the band that a row's state drops: the row that holds or makes one has
scale NaN and zero codes all the same, and the other rows are as without it."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from gpu_util import assert_bits, dev, host
from oracle import layer as L
from test_gpu_norm import Case

pytestmark = pytest.mark.gpu
M = 13
STATE = (np.arange(M) % 2).astype(np.uint8)            # odd rows are masked


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("center", [False, True], ids=["rms", "centred"])
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
@pytest.mark.parametrize("K,dm,du", [(64, 5, 11), (576, 18, 18), (1088, 8, 16), (4096, 128, 128), (8256, 1, 300),
                                     (18944, 592, 592)])
def test_scale_is_nan(K, dm, du, f32, center, bits):
    rng = np.random.default_rng(K)
    c = Case(rng, M, K, f32, mod=True, seqs=3)
    c.seq = np.zeros(M, np.int32)
    m_band, u_band = K - du - dm, K - du               # what unmasked and masked rows drop begins here
    c.h[2, u_band - 1], c.h[4, m_band] = np.inf, np.nan
    c.h[3, u_band], c.h[5, K - 1] = -np.inf, np.nan
    c.y[6, m_band], c.y[7, K - 1] = -np.inf, np.inf
    c.h[8, m_band] = c.y[8, m_band] = 65504            # an infinity made by an fp16 sum, not by an fp32 one
    c.kw["shift"][1, m_band], c.kw["shift"][2, u_band] = np.inf, -np.inf
    c.rows = dev(np.concatenate([np.zeros((3, K), np.float16), c.kw["scale"], c.kw["shift"]], 1))
    c.seq[10], c.seq[11] = 1, 2                        # conditions that are not finite, of one row each
    n, h = c.want(center=center)
    q, s = L.quantise_gated(n, STATE, dm, du, bits)
    bad = np.isnan(s)
    assert set(np.flatnonzero(bad)) == {2, 3, 4, 5, 6, 7, 10, 11} | (set() if f32 else {8})
    Aq, s_a, h2 = sq.norm_quant(dev(c.h), dev(c.y), state=dev(STATE), d_m=dm, d_u=du, bits=bits,
                                **c.device_kw(center=center))
    assert np.isnan(host(s_a)[bad]).all()
    assert_bits(host(s_a)[~bad], s[~bad], "scales")
    assert_bits(host(Aq), q, "codes")
    assert_bits(host(h2)[~bad], h[~bad], "h'")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("K", [64, 1088, 4096, 8256])
def test_scale_is_nan_without_conditions(K, bits):
    """The same of a plain RMS norm, whose rate of a row with an infinity is 0; a NaN beside a state that
    drops nothing of it, and rows without a state."""
    rng = np.random.default_rng(K)
    c = Case(rng, M, K)
    c.h[2, K - K // 32 - 1], c.y[3, K - 1], c.h[6, 0] = np.inf, -np.inf, np.inf
    for state in (STATE, None):
        n, _ = c.want()
        q, s = L.quantise_gated(n, state, K // 32, K // 32, bits)
        assert set(np.flatnonzero(np.isnan(s))) == {2, 3, 6}
        Aq, s_a, _ = sq.norm_quant(dev(c.h), dev(c.y), state=dev(state), bits=bits, **c.device_kw())
        assert np.isnan(host(s_a)[[2, 3, 6]]).all()
        keep = np.isfinite(s)
        assert_bits(host(s_a)[keep], s[keep], "scales")
        assert_bits(host(Aq), q, "codes")


@pytest.mark.parametrize("K", [64, 576, 4096])
def test_places_past_the_row_are_no_part_of_it(K):
    """Rows of one large value: centred, their entries are 0 while the mean times r passes fp32."""
    h = np.full((3, K), 3e38, np.float32)
    state = np.array([0, 1, 1], np.uint8)
    n, _ = L.norm(h, center=True)
    assert (n == 0).all()
    Aq, s_a, _ = sq.norm_quant(dev(h), state=dev(state), center=True)
    assert (host(s_a) == 0).all() and (host(Aq) == 0).all()
