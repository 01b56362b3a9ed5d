"""Every instance of the norm kernels bit for bit: shares of a row, types of the stream, with and without
options, out as rows or as codes of either width; and rows, streams, codes and conditions past 2^31."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from gpu_util import assert_bits, dev, host
from oracle import layer as L
from test_gpu_norm import Case, check

# (waves, vectors a lane): the shapes (rows, width) that take it
INSTANCES = {
    (1, 1): [(5, 448)], (2, 1): [(5, 576)], (4, 1): [(5, 1088)], (2, 2): [(1025, 1088)], (8, 1): [(5, 2112)],
    (4, 2): [(513, 2112)], (8, 2): [(5, 4160), (3, 5120), (3, 8192)], (16, 2): [(5, 8256)], (16, 4): [(3, 16448)],
}
SHAPES = [s for shapes in INSTANCES.values() for s in shapes]


@pytest.mark.gpu
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("full", [False, True], ids=["plain", "options"])
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
def test_instance(M, K, f32, full):
    rng = np.random.default_rng(M + K)
    c = Case(rng, M, K, f32, post=full, gate=full, mod=full, seqs=4 if full else 1)
    n, h = check(c, center=full)
    state = (rng.random(M) < 0.5).astype(np.uint8)
    for bits in (4, 8):
        q, s = L.quantise_gated(n, state, K // 32, K // 32, bits)
        Aq, s_a, h2 = sq.norm_quant(dev(c.h), dev(c.y), state=dev(state), bits=bits, **c.device_kw(center=full, alpha=0.5))
        assert_bits(host(Aq), q, (bits, "codes"))
        assert_bits(host(s_a), s, (bits, "scales"))
        assert_bits(host(h2), h, (bits, "h'"))


@pytest.mark.gpu
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
def test_stream_and_codes_past_31_bits(f32):
    """More than 2^31 entries of the stream in place, the block's output, the rows and their 8-bit codes: the
    last rows are those of a call of their own."""
    M, K = 70000, 32768
    g = torch.Generator(device="cuda").manual_seed(3)
    dtype = torch.float32 if f32 else torch.float16
    h = torch.zeros(M, K, dtype=dtype, device="cuda")
    y = torch.zeros(M, K, dtype=torch.float16, device="cuda")
    out = torch.full((M, K), 7.0, dtype=torch.float16, device="cuda")
    Aq = torch.full((M, K), 7, dtype=torch.int8, device="cuda")
    state = torch.zeros(M, dtype=torch.uint8, device="cuda")
    weight = (1 + 0.2 * torch.randn(K, generator=g, device="cuda")).to(torch.float16)
    h[-3:] = torch.randn(3, K, generator=g, device="cuda").to(dtype)
    y[-3:] = torch.randn(3, K, generator=g, device="cuda").to(torch.float16)
    state[-2] = 1
    kw = dict(weight=weight, alpha=0.5, bits=8)
    want_x = torch.empty(3, K, dtype=torch.float16, device="cuda")
    want = sq.norm_quant(h[-3:].clone(), y[-3:].clone(), state=state[-3:].clone(), out=want_x, **kw)
    _, s_a, h2 = sq.norm_quant(h, y, state=state, h_out=h, out=out, Aq=Aq, **kw)
    assert h2 is h
    for got, ref in ((Aq[-3:], want[0]), (s_a[-3:], want[1]), (h[-3:], want[2]), (out[-3:], want_x)):
        assert torch.equal(got, ref) and bool(ref.any())
    for t in (Aq, s_a, h, out):
        assert not bool(t[:1000].any()) and not bool(t[-1003:-3].any())


@pytest.mark.gpu
def test_conditions_past_31_bits():
    """Rows of gate, scale and shift that begin past 2^31 entries."""
    K, row = 520, 2 ** 30 + 8
    rng = np.random.default_rng(5)
    c = Case(rng, 7, K, True, post=True, gate=True, mod=True, seqs=3)
    far = torch.zeros(2 * row + 3 * K, dtype=torch.float16, device="cuda")
    view = far.as_strided((3, 3 * K), (row, 1))
    view.copy_(c.rows)
    c.rows, c.seq = view, np.array([2, 0, 1, 2, 2, 1, 0], np.int32)
    check(c, center=True)
