"""Every instance of the weight-only kernels: row tiles, groups of outputs, waves, rows read as operands
or in whole lines, each kind of scale group; few steps (waves without one) and many.

Tolerances: test_gpu_w4a16.py's for the product; the same sum behind a bias, in fp32: two more
roundings (the sum and Y)."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import dev, host, pack_codes
from oracle import attn as A
from oracle import frag as F
from oracle import layer as L
from test_gpu_w4a16 import check

# (tm, ng, waves, lines): M, N
INSTANCES = {
    (1, 1, 8, False): (4, 40), (1, 1, 8, True): (5, 40),
    (1, 2, 8, False): (1, 4104), (1, 2, 8, True): (8, 4120),
    (1, 2, 4, False): (1, 49160),
    (1, 3, 8, False): (3, 8200), (1, 3, 8, True): (11, 8216),
    (1, 3, 4, False): (4, 32776), (1, 3, 4, True): (7, 32776),
    (1, 4, 4, False): (1, 12296), (1, 4, 4, True): (13, 12312),
    (1, 5, 4, False): (3, 16392), (1, 5, 4, True): (16, 16424),
    (2, 1, 8, True): (17, 56), (2, 1, 4, True): (17, 8200),
    (2, 2, 8, True): (32, 4136), (2, 2, 4, True): (29, 8232),
    (4, 1, 4, True): (47, 72), (4, 2, 4, True): (130, 1384),
}


@pytest.mark.gpu
@pytest.mark.parametrize("group,K", [(32, 192), (64, 320), (128, 640), (256, 768)])
@pytest.mark.parametrize("name", INSTANCES, ids=lambda n: "-".join(map(str, n)))
def test_instance(name, group, K):
    M, N = INSTANCES[name]
    if N < 10000:
        K = 9 * K if group > 32 else 5 * K
    rng = np.random.default_rng(M + N + K)
    codes = rng.integers(-8, 8, (N, K), dtype=np.int8)
    s = (rng.uniform(0.5, 1.5, (K // group, N)) * 0.2 / K ** 0.5).astype(np.float16)
    X, bias = normal(rng, M, K), normal(rng, N)
    x, w, scale = dev(X), dev(F.to_frag(pack_codes(codes), K)), dev(s)
    Y = torch.full((M + 1, N), 7.0, dtype=torch.float16, device="cuda")
    check(sq.w4a16_gemm_frag(x, w, scale, Y=Y[:M]), X, codes, s, group)
    assert (host(Y)[M] == 7).all()
    t, mass = A.w4a16(X, codes, s, group)
    b = bias.astype(np.float64)
    got = host(sq.w4a16_linear(x, w, scale, bias=dev(bias), dtype=torch.float32)).astype(np.float64)
    tol = (K + 4) * L.U * mass + (np.abs(t) + np.abs(b)) * 2 * L.U + 2.0 ** -126
    assert (np.abs(got - (t + b)) <= tol).all(), float((np.abs(got - (t + b)) / tol).max())
