"""Norms with the residual stream, and the quantiser behind them, bit for bit: sums in fp64
are rounded once to fp32, everything else is single fp32 operations."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import normal
from gpu_util import assert_bits, dev, host
from oracle import layer as L

pytestmark = pytest.mark.gpu

KS = (8, 16, 64, 504, 512, 520, 1032, 2048, 2056, 3584, 4096, 4104, 8192, 8200, 16384, 16392, 18944, 32760, 32768)


class Case:
    def __init__(self, rng, M, K, f32=False, add=True, post=False, gate=False, mod=False, seqs=1, weight=True):
        h = rng.normal(0, 1, (M, K))
        h[:, 3::97] *= 12
        self.M, self.K = M, K
        self.h = h.astype(np.float32 if f32 else np.float16)
        self.y = normal(rng, M, K) if add else None
        self.kw = {}
        if weight:
            self.kw["weight"] = (1 + normal(rng, K, scale=0.2)).astype(np.float16)
        if add and post:
            self.kw["post_weight"] = (1 + normal(rng, K, scale=0.2)).astype(np.float16)
        rows = normal(rng, seqs, 3 * K, scale=0.3)
        if add and gate:
            self.kw["gate"] = rows[:, :K]
        if mod:
            self.kw["scale"], self.kw["shift"] = rows[:, K:2 * K], rows[:, 2 * K:]
        self.rows = dev(rows)
        self.seq = rng.integers(0, seqs, M).astype(np.int32) if seqs > 1 else None

    def device_kw(self, **kw):
        """Keyword arguments as device tensors, gate, scale and shift as views of one projection's rows."""
        out = {k: dev(v) for k, v in self.kw.items() if k not in ("gate", "scale", "shift")}
        for i, k in enumerate(("gate", "scale", "shift")):
            if k in self.kw:
                out[k] = self.rows[:, i * self.K:(i + 1) * self.K]
        if self.seq is not None:
            out["seq"] = dev(self.seq)
        return {**out, **kw}

    def want(self, **kw):
        return L.norm(self.h, self.y, seq=self.seq, **self.kw, **kw)


def check(c, center=False, alpha=0.5, eps=1e-6):
    n, h = c.want(center=center, alpha=alpha, eps=eps)
    hd, yd = dev(c.h), dev(c.y)
    out = torch.full((c.M + 1, c.K), 7.0, dtype=torch.float16, device="cuda")
    X, h2 = sq.norm(hd, yd, **c.device_kw(center=center, alpha=alpha, eps=eps, out=out[:-1]))
    with np.errstate(over="ignore"):
        assert_bits(host(X), n.astype(np.float16), "X")
    assert_bits(host(h2), h, "h'")
    assert (h2 is hd) == (c.y is None) and (host(out)[-1] == 7).all()
    assert_bits(host(hd), c.h, "h untouched")
    if c.y is not None:                                # the stream in place
        X2, h3 = sq.norm(hd, yd, **c.device_kw(center=center, alpha=alpha, eps=eps, h_out=hd))
        assert h3 is hd
        assert_bits(host(X2), host(X), "X, in place")
        assert_bits(host(hd), h, "h', in place")
    return n, h


@pytest.mark.parametrize("K", KS)
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
def test_widths(K, f32):
    rng = np.random.default_rng(K)
    check(Case(rng, 5, K, f32))
    check(Case(rng, 3, K, f32, post=True, gate=True, mod=True, seqs=4), center=True)


@pytest.mark.parametrize("K", [1032, 2048, 2056, 4096])
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
def test_many_rows_of_middle_widths(K, f32):
    """More rows than the plan's borders, which take another share of a row a wave."""
    rng = np.random.default_rng(K)
    M = 1100
    c = Case(rng, M, K, f32, post=True, gate=True, mod=True, seqs=4)
    check(c, center=True)
    c = Case(rng, M, K, f32)
    n, h = check(c)
    state = (rng.random(M) < 0.5).astype(np.uint8)
    if K % 64 == 0:
        for bits in (4, 8):
            q, s = L.quantise(L.gated(n, state, K // 32, K // 32), bits)
            Aq, s_a, _ = sq.norm_quant(dev(c.h), dev(c.y), state=dev(state), bits=bits, **c.device_kw(alpha=0.5))
            assert_bits(host(Aq), q, "codes")
            assert_bits(host(s_a), s, "scales")


@pytest.mark.parametrize("M,K", [(5, 520), (5, 4096), (600, 4096), (5, 20000)])
@pytest.mark.parametrize("spread", [2.0 ** -9, 2.0 ** -4, 0.26, 1.0])
def test_means_far_from_zero(M, K, spread):
    """Rows whose mean is many times their spread: the sum of squares takes a second pass there."""
    rng = np.random.default_rng(K)
    c = Case(rng, M, K, True, post=True)
    c.h = (1 + spread * rng.normal(0, 1, (M, K))).astype(np.float32)
    c.h[0] = 1.0
    c.y = (1 + spread * rng.normal(0, 1, (M, K))).astype(np.float16)
    check(c, center=True)


OPTIONS = [dict(), dict(add=False), dict(weight=False), dict(post=True), dict(gate=True), dict(gate=True, seqs=5),
           dict(mod=True, seqs=3), dict(mod=True, add=False), dict(post=True, gate=True, mod=True, seqs=7),
           dict(add=False, weight=False)]


@pytest.mark.parametrize("o", OPTIONS, ids=[" ".join(f"{k}={v}" for k, v in o.items()) or "plain" for o in OPTIONS])
@pytest.mark.parametrize("center", [False, True], ids=["rms", "centred"])
@pytest.mark.parametrize("f32", [False, True], ids=["fp16", "fp32"])
@pytest.mark.parametrize("M,K", [(1, 4096), (17, 520), (6, 8), (2, 8200)])
def test_options(M, K, o, center, f32):
    check(Case(np.random.default_rng(M + K), M, K, f32, **o), center, alpha=-0.75, eps=1e-3)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("K", [64, 128, 576, 2048, 3584, 4096, 8256, 18944, 32768])
def test_codes(K, bits):
    rng = np.random.default_rng(K + bits)
    for f32, o, center in ((False, {}, False), (True, dict(post=True, gate=True, mod=True, seqs=3), True),
                           (False, dict(add=False), False)):
        c = Case(rng, 9, K, f32, **o)
        state = (rng.random(9) < 0.5).astype(np.uint8)
        for st, dm, du in ((state, None, None), (None, None, None), (state, 5, K // 2), (state, 0, 0), (state * 3, 0, 11)):
            n, h = c.want(center=center, alpha=0.5)
            a, b = (K // 32 if x is None else x for x in (dm, du))
            q, s = L.quantise(L.gated(n, st, a, b), bits)
            out = torch.empty(9, K, dtype=torch.float16, device="cuda")
            Aq, s_a, h2 = sq.norm_quant(dev(c.h), dev(c.y), state=dev(st), d_m=dm, d_u=du, bits=bits, out=out,
                                        **c.device_kw(center=center, alpha=0.5))
            assert_bits(host(s_a), s, "scales")
            assert_bits(host(Aq), q, "codes")
            assert_bits(host(h2), h, "h'")
            assert_bits(host(out), n.astype(np.float16), "X")
            Aq2, s2, _ = sq.norm_quant(dev(c.h), dev(c.y), state=dev(st), d_m=dm, d_u=du, bits=bits,
                                       **c.device_kw(center=center, alpha=0.5))
            assert_bits(host(Aq2), q, "codes alone")
            assert_bits(host(s2), s, "scales alone")


def test_codes_feed_the_product():
    """The codes are those of the quantiser's own call on the fp32 rows, state gate aside."""
    rng = np.random.default_rng(1)
    c = Case(rng, 33, 512)
    n, _ = c.want(alpha=1.0)
    Aq, s_a, _ = sq.norm_quant(dev(c.h), dev(c.y), **c.device_kw())
    rq, rs = sq.sgat_quantize(dev(n))
    assert_bits(host(Aq), host(rq), "codes")
    assert_bits(host(s_a), host(rs), "scales")


def test_extremes():
    """Zero rows, constant rows, the largest and smallest values of fp16 and fp32."""
    K = 1032
    h = np.zeros((8, K), np.float16)
    h[1], h[2], h[3] = 1.0, 65504, 6e-8
    h[4, ::2] = -65504
    h[5, 7] = 65504
    h[6] = np.linspace(-1, 1, K)
    for center in (False, True):
        for eps in (1e-6, 1e-12, 1e-30, 10.0):
            n, _ = L.norm(h, eps=eps, center=center)
            X, _ = sq.norm(dev(h), eps=eps, center=center)
            assert_bits(host(X), n.astype(np.float16), (center, eps))
    g = h.astype(np.float32)
    g[2], g[3], g[4, ::2] = 1e30, 1e-30, -3e38
    n, _ = L.norm(g, eps=1e-6)
    X, _ = sq.norm(dev(g))
    with np.errstate(over="ignore"):
        assert_bits(host(X), n.astype(np.float16), "fp32")
    q, s = L.quantise(np.zeros((1, 64), np.float32), 4)
    Aq, s_a, _ = sq.norm_quant(torch.zeros(1, 64, dtype=torch.float16, device="cuda"))
    assert host(s_a)[0] == 0 and (host(Aq) == 0).all()


@pytest.mark.parametrize("K", [64, 4096, 8256])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_non_finite_rows_stay_alone(K, value):
    rng = np.random.default_rng(K)
    c = Case(rng, 9, K)
    clean = [host(t) for t in sq.norm_quant(dev(c.h), dev(c.y), bits=8, **c.device_kw())]
    clean_x = host(sq.norm(dev(c.h), dev(c.y), **c.device_kw())[0])
    c.h[2, K // 3] = value
    c.y[7, K - 1] = value
    Aq, s_a, h2 = sq.norm_quant(dev(c.h), dev(c.y), bits=8, **c.device_kw())
    X, _ = sq.norm(dev(c.h), dev(c.y), **c.device_kw())
    keep = np.ones(9, bool)
    keep[[2, 7]] = False
    assert np.isnan(host(s_a)[~keep]).all() and (host(Aq)[~keep] == 0).all()
    assert_bits(host(s_a)[keep], clean[1][keep], "scales")
    assert_bits(host(Aq)[keep], clean[0][keep], "codes")
    assert_bits(host(X)[keep], clean_x[keep], "X")
    assert np.isnan(host(X)[2, K // 3]) and np.isnan(host(X)[7, K - 1])


def test_rows_of_conditions_out_of_range():
    """Indexes outside the rows take the nearest; a single row needs none."""
    rng = np.random.default_rng(2)
    c = Case(rng, 6, 520, gate=True, mod=True, seqs=3)
    c.seq = np.array([-5, 0, 1, 2, 3, 2 ** 31 - 1], np.int32)
    check(c)
    one = Case(rng, 6, 520, gate=True, mod=True)
    n, h = one.want(alpha=1.0)
    kw = one.device_kw()
    for k in ("gate", "scale", "shift"):
        kw[k] = kw[k][0].clone()                        # [K]
    X, h2 = sq.norm(dev(one.h), dev(one.y), **kw)
    assert_bits(host(X), n.astype(np.float16), "X")
    assert_bits(host(h2), h, "h'")


def test_many_rows_and_empty():
    rng = np.random.default_rng(4)
    h = np.repeat(rng.normal(0, 1, (7, 64)).astype(np.float16), 20001, 0)
    X, _ = sq.norm(dev(h))
    n, _ = L.norm(h[::20001])
    assert_bits(host(X), np.repeat(n.astype(np.float16), 20001, 0), "140007 rows")
    X, h2 = sq.norm(dev(h[:0]), dev(h[:0]))
    assert X.shape == (0, 64) and h2.shape == (0, 64)
    Aq, s, _ = sq.norm_quant(dev(h[:0]))
    assert Aq.shape == (0, 32) and s.shape == (0,)


def test_offsets_past_31_bits():
    """Rows of the stream whose bytes begin past 2^31 and entries past 2^31 (fp32 and fp16)."""
    M, K = 70000, 32768
    h = torch.zeros(M, K, dtype=torch.float16, device="cuda")
    h[-3:] = torch.arange(3 * K, device="cuda").view(3, K).remainder(37).to(torch.float16)
    want = sq.norm(h[-3:].clone())[0]
    X, _ = sq.norm(h, out=torch.empty_like(h))
    assert torch.equal(X[-3:], want) and not bool(X[:100].any())
    del X, h


@pytest.mark.parametrize("shared", ["gate", "scale", "shift"])
def test_one_row_among_rows_of_conditions(shared):
    """A layer's own row with per-sequence ones, as [K], as [1, K] and as a view that repeats it."""
    rng = np.random.default_rng(3)
    c = Case(rng, 9, 520, gate=True, mod=True, post=True, seqs=4)
    kw = c.device_kw(alpha=0.5)
    row = kw[shared][1]
    c.kw[shared] = np.repeat(c.kw[shared][1:2], 4, 0)
    n, h = c.want(alpha=0.5)
    for form in (row.clone(), row.clone()[None], row.clone()[None].expand(4, -1)):
        X, h2 = sq.norm(dev(c.h), dev(c.y), **{**kw, shared: form})
        assert_bits(host(X), n.astype(np.float16), "X")
        assert_bits(host(h2), h, "h'")
    with pytest.raises(ValueError):
        sq.norm(dev(c.h), dev(c.y), **{**kw, shared: row[None].expand(3, -1)})
    with pytest.raises(ValueError):
        sq.norm(dev(c.h), dev(c.y), **{**kw, "seq": None})
