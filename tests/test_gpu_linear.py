"""Products with bias, activation, gate and residual in their epilogue.

t, bias, relu, gates and residual are single fp32 operations on exact int32 sums: bit for
bit.  silu and the gelus: within the bound of their steps (oracle/layer.py)."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import assert_bits, dev, host, pack_codes
from linear_cases import FRAGMENTS, GLU_SHAPES, Product, check, guarded
from oracle import attn as A
from oracle import frag as F
from oracle import layer as L

pytestmark = pytest.mark.gpu
NAN, INF = np.nan, np.inf


@pytest.mark.parametrize("glu", [False, True], ids=["plain", "glu"])
@pytest.mark.parametrize("name", FRAGMENTS)
def test_every_kernel(name, glu):
    """Each kernel a call can take, ragged: bias, activation and a residual, in place or not."""
    M, N, K = (GLU_SHAPES if glu else FRAGMENTS)[name]
    rng = np.random.default_rng(M + N + K + glu)
    p = Product(rng, int(name[0]), M, N, K, glu)
    bias = normal(rng, N)
    t = L.dequantised(p.acc, p.s_a, p.s_w, bias)
    r16, r32 = normal(rng, *p.out()), rng.normal(0, 1, p.out()).astype(np.float32)
    check(p.linear(bias=bias, act="relu", residual=r16), t, "relu", glu, r16, "fp16")
    Y = guarded(p.out(), torch.float32, r32)
    check(p.linear(bias=bias, act="silu", residual=Y[:-1], Y=Y[:-1]), t, "silu", glu, r32, "fp32 in place")
    assert (host(Y)[-1] == 7).all()
    Y = guarded(p.out(), torch.float16)
    check(p.linear(Y=Y[:-1]), L.dequantised(p.acc, p.s_a, p.s_w), "none", glu, None, "nothing but the product")
    assert (host(Y)[-1] == 7).all()
    if not glu:
        assert_bits(host(Y)[:-1], host(p.gemm(p.plain)), "the plain product")


@pytest.mark.parametrize("act", sq.ACTIVATIONS)
@pytest.mark.parametrize("glu", [False, True], ids=["plain", "glu"])
@pytest.mark.parametrize("bits,M,N,K", [(4, 1, 1024, 512), (4, 40, 512, 256), (4, 300, 1216, 64), (8, 3, 256, 320),
                                        (8, 130, 12176, 64)])
def test_activations(act, glu, bits, M, N, K):
    rng = np.random.default_rng(M + N)
    p = Product(rng, bits, M, N, K, glu)
    p.s_w *= 3
    bias = normal(rng, N)
    t = L.dequantised(p.acc, p.s_a, p.s_w, bias)
    for dtype, np_dtype in ((torch.float16, np.float16), (torch.float32, np.float32)):
        res = rng.normal(0, 1, p.out()).astype(np_dtype)
        check(p.linear(bias=bias, act=act, dtype=dtype), t, act, glu, None, (act, dtype))
        check(p.linear(bias=bias, act=act, residual=res), t, act, glu, res, (act, dtype, "residual"))
        check(p.linear(act=act, dtype=dtype), L.dequantised(p.acc, p.s_a, p.s_w), act, glu, None, (act, dtype, "no bias"))


@pytest.mark.parametrize("act", sq.ACTIVATIONS)
def test_activation_range(act):
    """One product of 1 a column: t is the column's scale, over the range of fp32."""
    N, K = 4096, 64
    A_, W = np.zeros((1, K // 2), np.uint8), np.zeros((N, K // 2), np.uint8)
    A_[0, 0], W[:, 0] = 1, 1
    t = np.concatenate([np.linspace(-30, 30, 3000), np.logspace(-40, 2, 540), -np.logspace(-40, 2, 540),
                        np.zeros(16)]).astype(np.float32)
    t[-16:] = [0.0, -0.0, 1e4, -1e4, 1e19, -1e19, 3e38, -3e38, 1e-45, -1e-45, 88.8, -88.8, 104.5, -104.5, -14.9, 9.0]
    Y = sq.w4a4_linear(dev(A_), dev(np.ones(1, np.float32)), sq.weights_to_frag(dev(W)), dev(t), act=act,
                       dtype=torch.float32)
    check(Y, t[None], act, False, None, act)


def test_non_finite():
    """NaN and infinities of scales, bias and residual stay in their row and column."""
    rng = np.random.default_rng(5)
    for M in (5, 70):
        p = Product(rng, 4, M, 64, 128, True)
        bias, res = normal(rng, 64), normal(rng, M, 32)
        clean = host(p.linear(bias=bias, act="silu", residual=res))
        bias[3], bias[32 + 9], res[2, 20] = NAN, INF, NAN
        p.s_a[4] = NAN
        got = host(p.linear(bias=bias, act="silu", residual=res))
        bad = np.zeros((M, 32), bool)
        bad[4] = bad[:, 3] = bad[2, 20] = True
        assert np.isnan(got[bad]).all()
        assert (np.isinf(got[:, 9]) | np.isnan(got[:, 9])).all()
        bad[:, 9] = True
        assert_bits(got[~bad], clean[~bad], "the others")


def test_overflow_to_infinity_and_largest_sums():
    """fp16 outputs past 65504 are infinite; K = 131072 of -8 by -8, whose scaled sum wraps."""
    K = 131072
    A_, W = np.full((20, K // 2), 0x88, np.uint8), np.full((32, K // 2), 0x88, np.uint8)
    for M in (1, 20):
        s = np.ones(32, np.float32)
        Y = sq.w4a4_linear(dev(A_[:M]), dev(np.ones(M, np.float32)), sq.weights_to_frag(dev(W)), dev(s),
                           dtype=torch.float32)
        assert (host(Y) == 64.0 * K).all()
        Y = sq.w4a4_linear(dev(A_[:M]), dev(np.ones(M, np.float32)), sq.weights_to_frag(dev(W), glu=True), dev(s), glu=True)
        assert np.isposinf(host(Y)).all()


@pytest.mark.parametrize("N,K", [(16, 64), (48, 192), (1040, 320)])
def test_fragments_of_pairs(N, K):
    rng = np.random.default_rng(N)
    Wq = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
    assert_bits(host(sq.weights_to_frag(dev(Wq), glu=True)), F.to_frag(L.paired_rows(Wq), K), "4-bit")
    W8 = rng.integers(-128, 128, (N, K)).astype(np.int8)
    assert_bits(host(sq.weights_to_frag(dev(W8), glu=True)), F.to_frag(L.paired_rows(W8).view(np.uint8), 2 * K), "8-bit")


# ---- weight-only -----------------------------------------------------------------------------------------

W4_SHAPES = [(1, 16, 64, 32), (1, 4096, 512, 128), (3, 48, 320, 32), (16, 528, 1024, 128), (17, 272, 1152, 384),
             (33, 80, 2048, 1024), (64, 144, 640, 640), (65, 16, 256, 128), (130, 1040, 576, 32), (2, 12288, 512, 64),
             (1, 24576, 256, 32), (16, 37888, 192, 64), (9, 24592, 384, 128), (1, 16400, 512, 512), (16, 61456, 128, 64),
             (17, 8208, 192, 64), (64, 12304, 128, 32), (31, 16400, 128, 128), (12, 20496, 320, 32)]


@pytest.mark.parametrize("M,N,K,group", W4_SHAPES)
@pytest.mark.parametrize("glu,act,res", [(False, "none", "f32"), (True, "silu", None), (True, "gelu", "f16"),
                                         (False, "relu2", "f16")])
def test_weight_only(M, N, K, group, glu, act, res):
    rng = np.random.default_rng(M + N + K)
    codes = rng.integers(-8, 8, (N, K))
    s = (rng.uniform(0.5, 1.5, (K // group, N)) * 0.2 / K ** 0.5).astype(np.float16)
    X, bias = normal(rng, M, K), normal(rng, N)
    W = pack_codes(codes)
    Wf = dev(F.to_frag(L.paired_rows(W) if glu else W, K))
    t, mass = A.w4a16(X, codes, s, group)
    b = bias.astype(np.float64)
    err = (K + 4) * L.U * mass + (np.abs(t) + np.abs(b)) * L.U
    dtype = np.float32 if res == "f32" else np.float16
    out = (M, N // 2 if glu else N)
    r = None if res is None else rng.normal(0, 1, out).astype(dtype)
    Y = guarded(out, torch.float32 if res == "f32" else torch.float16, r)
    got = sq.w4a16_linear(dev(X), Wf, dev(s), bias=dev(bias), act=act, glu=glu, Y=Y[:-1],
                          residual=None if r is None else Y[:-1])
    y, bound = L.epilogue(t + b, act, glu, r, err, dtype)
    off = np.abs(host(got).astype(np.float64) - y)
    assert (off <= bound).all(), float((off / bound).max())
    assert (host(Y)[-1] == 7).all()
    if not glu:
        assert_bits(host(sq.w4a16_linear(dev(X), Wf, dev(s))), host(sq.w4a16_gemm_frag(dev(X), Wf, dev(s))), "plain")


def test_empty():
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    f = torch.float32
    assert sq.w4a4_linear(z(0, 64), z(0, dt=f), z(1, 2, 1024), z(32, dt=f), glu=True, act="silu").shape == (0, 16)
    assert sq.w4a4_linear(z(3, 64), z(3, dt=f), z(1, 0, 1024), z(0, dt=f), dtype=f).shape == (3, 0)
    assert sq.w4a16_linear(z(0, 128, dt=torch.float16), z(1, 1, 1024), z(2, 16, dt=torch.float16)).shape == (0, 16)


@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
def test_offsets_past_31_bits(f32):
    """Outputs and residuals of more than 2^31 entries: the last rows are those of a call of their own."""
    M, N, K = 140001, 16400, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    byte = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    A_, W = byte(M, K // 2), byte(N, K // 2)
    s_a, s_w = (torch.rand(n, generator=g, device="cuda") * 0.1 + 0.01 for n in (M, N))
    bias = torch.randn(N, generator=g, device="cuda").to(torch.float16)
    dtype = torch.float32 if f32 else torch.float16
    tail = torch.randn(300, N, generator=g, device="cuda").to(dtype)
    Y = torch.zeros(M, N, device="cuda", dtype=dtype)
    Y[-300:] = tail
    Wf = sq.weights_to_frag(W)
    got = sq.w4a4_linear(A_, s_a, Wf, s_w, bias=bias, act="relu", residual=Y, Y=Y)
    for rows, res in ((slice(-300, None), tail), (slice(0, 300), None), (slice(65536 - 40, 65536 + 260), None)):
        want = sq.w4a4_linear(A_[rows].clone(), s_a[rows].clone(), Wf, s_w, bias=bias, act="relu", residual=res,
                              dtype=dtype)
        assert torch.equal(got[rows], want)
    del Y, got
