"""Weights that are not finite: the group's scale says so and its products are NaN."""
import numpy as np
import pytest

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import assert_bits, dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,group", [(64, 32), (192, 64), (512, 256)])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_groups_tell(K, group, value):
    rng = np.random.default_rng(K)
    W = normal(rng, 40, K, scale=0.05)
    W[3, group - 1] = value
    W[39, 0] = value
    Wq, s = sq.quantize_weights_group(dev(W), group)
    codes, want = A.quantize_group(W, group)
    got = host(Wq)
    low, high = (got & 15).astype(np.int64), (got >> 4).astype(np.int64)
    q = np.stack([low, high], -1).reshape(40, K)
    assert_bits(np.where(q > 7, q - 16, q), codes, "codes")
    assert np.array_equal(host(s), want, equal_nan=True)
    bad = [3, 39]
    assert not np.isfinite(want[0, bad]).any() and np.isfinite(np.delete(want, bad, 1)).all()
    y = host(sq.w4a16_gemm_frag(dev(normal(rng, 5, K)), sq.weights_to_frag(Wq), s))
    assert np.isnan(y[:, bad]).all() and np.isfinite(np.delete(y, bad, 1)).all()
