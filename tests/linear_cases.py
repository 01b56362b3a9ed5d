"""Shapes, inputs and comparisons of the products with a fused epilogue."""
import numpy as np
import torch

import paper_2606_04945_amd as sq
from gemm_kernels import KERNELS
from gpu_util import assert_bits, dev, host
from oracle import layer as L

FRAGMENTS = {name: shape for name, shape in KERNELS.items() if "fragments" in name}
# gated products have N % 16 == 0: the next multiple takes the same kernel but here
GLU_SHAPES = {name: (M, -(-N // 16) * 16, K) for name, (M, N, K) in FRAGMENTS.items()}


class Product:
    """Codes and scales on the device, weights in both orders, and the exact int32 sums by the plain
    product (whose own tests hold it to the oracle)."""

    def __init__(self, rng, bits, M, N, K, glu):
        top = 128 if bits == 8 else 8
        self.bits, self.glu, self.M, self.N = bits, glu, M, N
        a = torch.from_numpy(rng.integers(-top, top, (M, K)).astype(np.int8)).cuda()
        w = torch.from_numpy(rng.integers(-top, top, (N, K)).astype(np.int8)).cuda()
        if bits == 4:
            a, w = (x.view(torch.uint8) & 15 for x in (a, w))
            a, w = (x[:, 0::2] | (x[:, 1::2] << 4) for x in (a, w))
        self.A, W = a, w.contiguous()
        # t of order 1
        self.s_a = rng.uniform(0.5, 1.5, M).astype(np.float32)
        self.s_w = (rng.uniform(0.5, 1.5, N) * 3 / (top * top * K ** 0.5)).astype(np.float32)
        self.Wf = sq.weights_to_frag(W, glu=glu)
        plain = sq.weights_to_frag(W) if glu else self.Wf
        self.acc = host(self.gemm(plain, want_Y=False, want_acc=True)[1])
        self.plain = plain

    def gemm(self, Wf, **kw):
        return (sq.w8a8_gemm_frag if self.bits == 8 else sq.w4a4_gemm_frag)(self.A, dev(self.s_a), Wf, dev(self.s_w), **kw)

    def linear(self, **kw):
        kw = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
        return (sq.w8a8_linear if self.bits == 8 else sq.w4a4_linear)(self.A, dev(self.s_a), self.Wf, dev(self.s_w),
                                                                      glu=self.glu, **kw)

    def out(self):
        return self.M, self.N // 2 if self.glu else self.N


def check(got, t, act, glu, residual, what, dtype=None):
    """Bits where fp32 arithmetic fixes them, else the bound of the activation's steps."""
    got = host(got)
    dtype = got.dtype.type if dtype is None else dtype
    if act in L.EXACT:
        assert_bits(got, L.exact(t, act, glu, residual, dtype), what)
        return
    y, bound = L.epilogue(t, act, glu, residual, None, dtype)
    off = np.abs(got.astype(np.float64) - y)
    assert got.shape == y.shape and (off <= bound).all(), (what, float((off / bound).max()))


def guarded(shape, dtype, residual=None):
    """An output with a row of sevens behind it (and the residual in it, for calls in place)."""
    full = torch.full((shape[0] + 1, shape[1]), 7.0, dtype=dtype, device="cuda")
    if residual is not None:
        full[:-1] = dev(residual)
    return full
