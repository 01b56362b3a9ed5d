"""A layer's step without its attention, as a serving loop calls it:

  norm into codes -> fused projection with bias -> (stands for the attention: its first columns) ->
  TAC quantiser -> O projection onto the stream -> norm into codes -> gated gate + up product ->
  quantiser -> down product onto the stream -> the next layer's norm,

stage by stage against the oracle on the stage's own inputs; captured and replayed with new
tokens; on another stream than the current one; two at once on two streams."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import assert_bits, dev, host
from linear_cases import check
from oracle import layer as L
from oracle import oracle as O

pytestmark = pytest.mark.gpu

H, QKV, F = 512, 768, 704


def prepared(rng, N, K, glu=False):
    W = normal(rng, N, K, scale=K ** -0.5)
    Wq, s = sq.sgat_prepare_weights(dev(W))
    return sq.weights_to_frag(Wq, glu=glu), s, host(Wq)


class Layer:
    def __init__(self, seed, f32):
        rng = np.random.default_rng(seed)
        self.f32 = f32
        self.qkv, self.s_qkv, self.qkv_q = prepared(rng, QKV, H)
        self.o, self.s_o, self.o_q = prepared(rng, H, H)
        self.up, self.s_up, self.up_q = prepared(rng, 2 * F, H, glu=True)
        self.down, self.s_down, self.down_q = prepared(rng, H, F)
        self.bias = normal(rng, QKV, scale=0.3)
        self.w = [(1 + normal(rng, H, scale=0.1)).astype(np.float16) for _ in range(3)]
        self.rows = normal(rng, 3, 3 * H, scale=0.2)                  # gate, scale, shift of three sequences
        self.tac_M = (np.eye(16) + normal(rng, H // 16, 16, 16, scale=0.01)).astype(np.float16)
        self.tac_d = normal(rng, H, scale=0.01)
        self.d = {n: dev(getattr(self, n)) for n in ("bias", "rows", "tac_M", "tac_d")}
        self.dw = [dev(w) for w in self.w]

    def step(self, h, y, state, seq, stream=None):
        """One layer on the stream h and the previous block's output y."""
        d, kw = self.d, dict(stream=stream)
        gate, scale, shift = d["rows"][:, :H], d["rows"][:, H:2 * H], d["rows"][:, 2 * H:]
        A1, s1, h1 = sq.norm_quant(h, y, state=state, weight=self.dw[0], gate=gate, scale=scale, shift=shift, seq=seq, **kw)
        qkv = sq.w4a4_linear(A1, s1, self.qkv, self.s_qkv, bias=d["bias"], **kw)
        z = qkv[:, :H].contiguous() if stream is None else self._columns(qkv, stream)
        A2, s2 = sq.sgat_quant_act(z, state, None, None, None, d["tac_M"], d["tac_d"], 16, **kw)
        h2 = sq.w4a4_linear(A2, s2, self.o, self.s_o, residual=h1, Y=h1, **kw)          # in place
        A3, s3, _ = sq.norm_quant(h2, state=state, weight=self.dw[1], **kw)
        u = sq.w4a4_linear(A3, s3, self.up, self.s_up, act="silu", glu=True, **kw)
        A4, s4 = sq.sgat_quant_act(u, state, **kw)
        h3 = sq.w4a4_linear(A4, s4, self.down, self.s_down, residual=h2, **kw)
        x, _ = sq.norm(h3, weight=self.dw[2], **kw)
        return dict(A1=A1, s1=s1, qkv=qkv, A2=A2, s2=s2, h2=h2, A3=A3, s3=s3, u=u, A4=A4, s4=s4, h3=h3, x=x)

    @staticmethod
    def _columns(t, stream):
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))
        with torch.cuda.stream(s):
            return t[:, :H].contiguous()


def inputs(rng, M, f32):
    h, y = rng.normal(0, 1.5, (M, H)).astype(np.float32 if f32 else np.float16), normal(rng, M, H)
    return h, y, (rng.random(M) < 0.5).astype(np.uint8), rng.integers(0, 3, M).astype(np.int32)


def linear(A_, s_a, Wq, s_w, bias=None):
    acc = O.gemm(A_, s_a, Wq, s_w)[1]
    return L.dequantised(acc, s_a, s_w, bias)


@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
@pytest.mark.parametrize("M", [1, 19, 60, 300])
def test_stages(M, f32):
    layer, rng = Layer(1, f32), np.random.default_rng(M)
    h, y, state, seq = inputs(rng, M, f32)
    got = layer.step(dev(h), dev(y), dev(state), dev(seq))
    g = {k: host(v) for k, v in got.items()}
    dm, du = sq.default_band(H)
    r = layer.rows
    n, h1 = L.norm(h, y, layer.w[0], gate=r[:, :H], scale=r[:, H:2 * H], shift=r[:, 2 * H:], seq=seq)
    q, s = L.quantise(L.gated(n, state, dm, du), 4)
    assert_bits(g["A1"], q, "codes 1")
    assert_bits(g["s1"], s, "scales 1")
    check(got["qkv"], linear(q, s, layer.qkv_q, host(layer.s_qkv), layer.bias), "none", False, None, "qkv")
    rA, rs = O.quant_act(g["qkv"][:, :H].copy(), state, None, dm, du, layer.tac_M, layer.tac_d, 16)
    assert_bits(g["A2"], rA, "codes 2")
    check(got["h2"], linear(rA, rs, layer.o_q, host(layer.s_o)), "none", False, h1, "stream 2")
    n, _ = L.norm(g["h2"], weight=layer.w[1])
    q, s = L.quantise(L.gated(n, state, dm, du), 4)
    assert_bits(g["A3"], q, "codes 3")
    check(got["u"], linear(q, s, layer.up_q, host(layer.s_up)), "silu", True, None, "gated")
    fm, fu = sq.default_band(F)
    rA, rs = O.quant_act(g["u"], state, None, fm, fu)
    assert_bits(g["A4"], rA, "codes 4")
    check(got["h3"], linear(rA, rs, layer.down_q, host(layer.s_down)), "none", False, g["h2"], "stream 3")
    n, _ = L.norm(g["h3"], weight=layer.w[2])
    assert_bits(g["x"], n.astype(np.float16), "x")


@pytest.mark.parametrize("M", [3, 130])
def test_graph_replays_with_new_tokens(M):
    """One capture, replayed with other tokens in place, eager work in between."""
    layer, rng = Layer(3, True), np.random.default_rng(4)
    ins = [dev(a) for a in inputs(rng, M, True)]
    layer.step(*ins)
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            outs = layer.step(*ins)
    torch.cuda.synchronize()
    for n in range(5):
        for t, a in zip(ins, inputs(rng, M, True)):
            t.copy_(dev(a))
        want = {k: host(t).copy() for k, t in layer.step(*ins).items()}
        for t in outs.values():
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k, t in outs.items():
            assert_bits(host(t), want[k], f"replay {n}: {k}")


def test_other_stream_and_two_at_once():
    """On streams that are not the current one, by object and by handle, at the same time; shapes whose
    K split needs a workspace among them."""
    rng = np.random.default_rng(6)
    ins = [dev(a) for a in inputs(rng, 60, False)]
    want = [{k: host(t).copy() for k, t in Layer(seed, False).step(*ins).items()} for seed in (7, 8)]
    a, b = Layer(7, False), Layer(8, False)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got_a, got_b = a.step(*ins, stream=sa), b.step(*ins, stream=sb.cuda_stream)
    torch.cuda.synchronize()
    for got, w in ((got_a, want[0]), (got_b, want[1])):
        for k, t in got.items():
            assert_bits(host(t), w[k], k)
