"""Fused products whose K is split across workgroups (partial sums in a workspace, a second launch that
joins them and applies the epilogue): on other streams, two at once, captured and replayed."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import assert_bits, dev, host
from linear_cases import FRAGMENTS, GLU_SHAPES, Product, check
from oracle import layer as L

SPLIT = [name for name in FRAGMENTS if name.endswith("K split")]
CASES = [(name, glu) for name in SPLIT for glu in (False, True)]


class Step:
    """One product with bias, activation and an fp32 residual, and what it has to give."""

    def __init__(self, seed, name, glu):
        M, N, K = (GLU_SHAPES if glu else FRAGMENTS)[name]
        rng = np.random.default_rng(seed)
        self.p = Product(rng, int(name[0]), M, N, K, glu)
        assert sq.gemm_workspace_bytes(M, N, K, self.p.bits) > 0
        self.glu, self.res = glu, rng.normal(0, 1, self.p.out()).astype(np.float32)
        bias = normal(rng, N)
        self.t = L.dequantised(self.p.acc, self.p.s_a, self.p.s_w, bias)
        self.d = {k: dev(v) for k, v in dict(s_a=self.p.s_a, s_w=self.p.s_w, bias=bias, res=self.res).items()}

    def run(self, **kw):
        d, f = self.d, sq.w8a8_linear if self.p.bits == 8 else sq.w4a4_linear
        return f(self.p.A, d["s_a"], self.p.Wf, d["s_w"], bias=d["bias"], act="relu", glu=self.glu, residual=d["res"], **kw)

    def check(self, got, what):
        check(got, self.t, "relu", self.glu, self.res, what)


@pytest.mark.gpu
@pytest.mark.parametrize("name,glu", CASES, ids=str)
def test_two_streams_at_once(name, glu):
    """By stream object and by handle, workspaces of the calls' own and given ones."""
    a, b = Step(1, name, glu), Step(2, name, glu)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    n = sq.gemm_workspace_bytes(a.p.M, a.p.N, a.p.A.shape[1] * 8 // a.p.bits, a.p.bits)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for given in (None, ws):
        got = [(a.run(stream=sa, ws=given), b.run(stream=sb.cuda_stream)) for _ in range(4)]
        torch.cuda.synchronize()
        for n, (x, y) in enumerate(got):
            a.check(x, ("first stream", n, given is None))
            b.check(y, ("second stream", n, given is None))


@pytest.mark.gpu
@pytest.mark.parametrize("name,glu", CASES, ids=str)
def test_graph_replays_with_new_tokens(name, glu):
    """One capture of two products that follow each other, replayed with other codes in place, eager work
    in between."""
    a, b = Step(3, name, glu), Step(4, name, glu)
    a.check(a.run(), "eager")
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            outs = a.run(), b.run()
    torch.cuda.synchronize()
    new = torch.Generator(device="cuda").manual_seed(7)
    for n in range(4):
        for step in (a, b):
            step.p.A.view(torch.uint8).copy_(torch.randint(0, 256, step.p.A.shape, generator=new, device="cuda",
                                                           dtype=torch.uint8))
        want = [host(step.run()).copy() for step in (a, b)]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert_bits(host(t), w, f"replay {n}")


def test_the_cases_split():
    # (that these shapes take the kernels of their names: test_linear_plan.py)
    assert len(SPLIT) == 2 and {int(name[0]) for name in SPLIT} == {4, 8}
