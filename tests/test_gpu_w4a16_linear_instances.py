"""Every instance of the weight-only kernels: plain, and with a fused epilogue, gated and not, each with bias,
activation and a residual in place.

Tolerances: the product's of test_gpu_w4a16.py as an error of t, through the epilogue's bound of
oracle/layer.py."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import dev, host, pack_codes
from linear_cases import guarded
from oracle import attn as A
from oracle import frag as F
from oracle import layer as L
from test_gpu_w4a16_instances import INSTANCES

GROUPS = (32, 64, 256)


def shape(name, group):
    """(M, N, K) that takes instance `name` at scale groups of `group`.  N % 16 == 0 for gates: the next multiple is
    of as many groups of 16 outputs.  Rows are read in whole lines from some M and K on; half a last step where
    the group allows."""
    tm, ng, _, lines = name
    M, N = INSTANCES[name]
    N = -(-N // 16) * 16
    if tm == 1 and lines:
        K = {32: 1088 if ng == 1 else 3520 if ng < 4 else 2112, 64: 1088, 256: 1280}[group]
        return 16, N, K
    return M, N, {32: 192, 64: 320, 256: 768}[group] * (1 if N > 10000 else 9 if group > 32 else 5)


@pytest.mark.gpu
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("name", INSTANCES, ids=lambda n: "-".join(map(str, n)))
def test_instance(name, group):
    M, N, K = shape(name, group)
    rng = np.random.default_rng(M + N + K)
    codes = rng.integers(-8, 8, (N, K), dtype=np.int8)
    s = (rng.uniform(0.5, 1.5, (K // group, N)) * 0.2 / K ** 0.5).astype(np.float16)
    X, bias = normal(rng, M, K), normal(rng, N)
    t, mass = A.w4a16(X, codes, s, group)
    b = bias.astype(np.float64)
    err = (K + 4) * L.U * mass + (np.abs(t) + np.abs(b)) * L.U
    W = pack_codes(codes)
    Y = guarded((M, N), torch.float16)
    plain = host(sq.w4a16_gemm_frag(dev(X), dev(F.to_frag(W, K)), dev(s), Y=Y[:-1])).astype(np.float64)
    off = np.abs(plain - t) / (2.0 ** -11 * np.abs(t) + 2.0 ** -25 + (K + 4) * L.U * mass)
    assert (off <= 1).all() and (host(Y)[-1] == 7).all(), ("plain", float(off.max()))
    for glu, act, dtype in ((False, "gelu", np.float32), (True, "silu", np.float16)):
        out = (M, N // 2 if glu else N)
        r = rng.normal(0, 1, out).astype(dtype)
        Y = guarded(out, torch.float32 if dtype is np.float32 else torch.float16, r)
        got = sq.w4a16_linear(dev(X), dev(F.to_frag(L.paired_rows(W) if glu else W, K)), dev(s), bias=dev(bias), act=act,
                              glu=glu, residual=Y[:-1], Y=Y[:-1])
        y, bound = L.epilogue(t + b, act, glu, r, err, dtype)
        off = np.abs(host(got).astype(np.float64) - y)
        assert (off <= bound).all(), (act, float((off / bound).max()))
        assert (host(Y)[-1] == 7).all(), act
