"""The operators of a layer's attention side used together, as a serving loop calls them:

  weight-only QKV product -> rotation and append -> attention over the cache ->
  TAC, gate and 4-bit quantiser -> int4 O projection,

stage by stage against the oracle on the stage's own inputs, over several steps on one
cache; the whole step captured in a graph and replayed with new tokens and lengths; on
another stream than the current one; two calls at once on two streams."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import check_attention, normal
from gpu_util import assert_bits, dev, host
from oracle import attn as A
from oracle import oracle as O

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HKV, D, PAGE, B = 512, 8, 2, 64, 16, 3
QKV = (HQ + 2 * HKV) * D


class Layer:
    """Weights, cache and page table of one layer, on the device, and their oracle copies."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.W = normal(rng, QKV, HIDDEN, scale=0.05)
        self.Wq, self.s = sq.quantize_weights_group(dev(self.W), 64)
        self.Wf = sq.weights_to_frag(self.Wq)
        self.freq = sq.rope_frequencies(D, 1e4, scaling="yarn", factor=4.0, original=64.0)
        self.amp = sq.rope_amplitude("yarn", 4.0)
        self.cache = sq.kv_cache(40, HKV, D, PAGE)
        self.table = rng.permutation(40)[:B * 12].reshape(B, 12).astype(np.int32)
        self.tac_M = (np.eye(16) + normal(rng, HQ * D // 16, 16, 16, scale=0.01)).astype(np.float16)
        self.tac_d = normal(rng, HQ * D, scale=0.01)
        Wo = normal(rng, HIDDEN, HQ * D, scale=0.05)
        self.Woq, self.so = sq.sgat_prepare_weights(dev(Wo))
        self.Wof = sq.weights_to_frag(self.Woq)
        self.dev = {n: dev(getattr(self, n)) for n in ("table", "tac_M", "tac_d")}

    def step(self, x, state, cu, lens, causal, stream=None):
        d = self.dev
        qkv = sq.w4a16_gemm_frag(x, self.Wf, self.s, stream=stream)
        T = x.shape[0]
        q, k, v = (qkv[:, a * D:b * D].unflatten(1, (b - a, D))
                   for a, b in ((0, HQ), (HQ, HQ + HKV), (HQ + HKV, HQ + 2 * HKV)))
        q = sq.kv_append(self.cache, k, v, cu, lens, d["table"], freq=self.freq, amplitude=self.amp, q=q, stream=stream)
        z = sq.attn_kv8(q, self.cache, cu, lens, d["table"], causal=causal, stream=stream)
        Aq, s_a = sq.sgat_quant_act(z.view(T, HQ * D), state, None, None, None, d["tac_M"], d["tac_d"], 16,
                                    stream=stream)
        y = sq.w4a4_gemm_frag(Aq, s_a, self.Wof, self.so, stream=stream)
        return qkv, q, z, Aq, s_a, y


def batch(news, lens):
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    return dev(cu), dev(np.array(lens, np.int32)), cu, np.array(lens, np.int32)


def oracle_cache(layer):
    c = A.Cache(40, HKV, D, PAGE)
    c.k, c.v, c.ks, c.vs = (host(t) for t in layer.cache)
    return c


STEPS = [([20, 37, 9], [20, 37, 9], False), ([1, 1, 1], [21, 38, 10], True), ([16, 0, 16], [37, 38, 26], False),
         ([16, 0, 16], [37, 38, 26], False), ([1, 120, 2], [38, 158, 28], True)]


def test_steps_against_the_oracle():
    layer, rng = Layer(1), np.random.default_rng(2)
    for n, (news, lens, causal) in enumerate(STEPS):
        T = sum(news)
        x, state = normal(rng, T, HIDDEN), (rng.random(T) < 0.5).astype(np.uint8)
        cu_d, lens_d, cu, ln = batch(news, lens)
        before = oracle_cache(layer)
        qkv, q, z, Aq, s_a, y = layer.step(dev(x), dev(state), cu_d, lens_d, causal)
        codes, rs = A.quantize_group(layer.W, 64)
        want, mass = A.w4a16(x, codes, rs, 64)
        bound = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + (HIDDEN + 4) * 2.0 ** -24 * mass
        assert (np.abs(host(qkv) - want) <= bound).all()
        # queries, keys and values from the product's own bits
        h = host(qkv).reshape(T, HQ + 2 * HKV, D)
        pos = A.positions(cu, ln, T)
        freq = host(layer.freq)
        rq, rk = (A.rope(t, pos, freq, "half", layer.amp) for t in (h[:, :HQ], h[:, HQ:HQ + HKV]))
        size = layer.amp * np.abs(h[:, :HQ].astype(np.float64)).max()
        bound = 2.0 ** -11 * np.abs(rq) + 2.0 ** -25 + 2.0 ** -20 * size
        assert (np.abs(host(q) - rq) <= bound).all()
        A.append(before, rk, h[:, HQ + HKV:].astype(np.float32), cu, ln, layer.table)
        after = oracle_cache(layer)
        assert_bits(after.v, before.v, f"step {n}: values")
        assert_bits(after.vs, before.vs, f"step {n}: value scales")
        # keys within the rotation's error: a scale by 2^-20, a code by the step that its rounding may then take
        assert np.abs(after.k.astype(int) - before.k).max() <= 1
        assert np.allclose(after.ks, before.ks, rtol=2.0 ** -20, atol=0)
        check_attention(z, A.attention(host(q), after, cu, ln, layer.table, causal), f"step {n}")
        # the TAC quantiser and the O projection are bit-exact on the attention's output
        dm, du = sq.default_band(HQ * D)
        rA, rs_a = O.quant_act(host(z).reshape(T, -1), state, None, dm, du, layer.tac_M, layer.tac_d, 16)
        assert_bits(host(Aq), rA, "codes")
        assert_bits(host(s_a), rs_a, "scales")
        rY, _ = O.gemm(rA, rs_a, host(layer.Woq), host(layer.so))
        assert_bits(host(y), rY, "O projection")


def test_graph_replays_with_new_tokens():
    """One capture, replayed for steps whose tokens, lengths and pages change in place."""
    eager, graphed = Layer(3), Layer(3)
    rng = np.random.default_rng(4)
    x = torch.zeros(B, HIDDEN, dtype=torch.float16, device="cuda")
    state = torch.zeros(B, dtype=torch.uint8, device="cuda")
    cu, lens, _, _ = batch([1] * B, [1] * B)
    graphed.step(x, state, cu, lens, True)                       # warm-up; page slot 0 is written again below
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            outs = graphed.step(x, state, cu, lens, True)
    torch.cuda.synchronize()
    for n in range(40):                                          # lengths 1 .. 40: pages begin, fill and end
        x.copy_(dev(normal(rng, B, HIDDEN, scale=1 + n % 3)))
        state.copy_(dev((rng.random(B) < 0.5).astype(np.uint8)))
        lens.copy_(dev(np.array([n + 1, min(n + 1, 25), n + 1], np.int32)))
        want = [host(t).copy() for t in eager.step(x, state, cu, lens, True)]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for name, t, r in zip(("qkv", "q", "z", "Aq", "s_a", "y"), outs, want):
            assert_bits(host(t), r, f"replay {n}: {name}")
    for t, r in zip(graphed.cache, eager.cache):
        assert_bits(host(t), host(r), "cache")


@pytest.mark.parametrize("news,lens", [([1, 1], [3000, 40]), ([70, 80], [2500, 90]), ([20, 9], [2000, 1900])])
def test_split_attention_in_a_graph(news, lens):
    """Batches that are shared between workers and joined: captured, replayed with other lengths."""
    rng = np.random.default_rng(5)
    pages, page, heads, G, dim = 110, 64, 2, 4, 128
    cache = sq.KVCache(*(dev(t) for t in (rng.integers(-127, 128, (pages, heads, page, dim)).astype(np.int8),
                                         rng.integers(-127, 128, (pages, heads, dim, page)).astype(np.int8),
                                         rng.uniform(0.01, 0.02, (pages, heads)).astype(np.float32),
                                         rng.uniform(0.01, 0.02, (pages, heads)).astype(np.float32))))
    table = dev(rng.permutation(pages)[:104].reshape(2, 52).astype(np.int32))
    T = sum(news)
    q = dev(normal(rng, T, heads * G, dim))
    cu, ln, _, _ = batch(news, lens)
    call = lambda: sq.attn_kv8(q, cache, cu, ln, table, want_lse=True)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            out, lse = call()
    torch.cuda.synchronize()
    for n in range(4):
        q.copy_(dev(normal(rng, T, heads * G, dim)))
        ln.copy_(dev(np.array([lens[0] - 300 * n, lens[1] + 200 * n], np.int32)))
        want = [host(t).copy() for t in call()]
        out.fill_(5), lse.fill_(5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert_bits(host(out), want[0], f"replay {n}")
        assert_bits(host(lse), want[1], f"replay {n}: lse")


def test_other_stream_and_two_at_once():
    """On a stream that is not the current one, by object and by handle; two layers' steps at the same time."""
    rng = np.random.default_rng(6)
    x, st = dev(normal(rng, 66, HIDDEN)), dev((rng.random(66) < 0.5).astype(np.uint8))
    cu, lens, _, _ = batch([20, 37, 9], [20, 37, 9])
    want = [[host(t).copy() for t in Layer(seed).step(x, st, cu, lens, False)] for seed in (7, 8)]
    a, b = Layer(7), Layer(8)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):                                            # the same tokens again: nothing changes
        got_a = a.step(x, st, cu, lens, False, stream=sa)
        got_b = b.step(x, st, cu, lens, False, stream=sb.cuda_stream)
    torch.cuda.synchronize()
    for got, w in ((got_a, want[0]), (got_b, want[1])):
        for t, r in zip(got, w):
            assert_bits(host(t), r, "stream")
