"""The reference of epilogues and norms against formulas written another way."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import layer as L


def test_activations():
    t = np.linspace(-12, 12, 4001)
    x = torch.from_numpy(t)
    want = {"none": x, "relu": F.relu(x), "relu2": F.relu(x) ** 2, "silu": F.silu(x), "gelu": F.gelu(x),
            "gelu_tanh": F.gelu(x, approximate="tanh")}
    for act, y in want.items():
        assert np.allclose(L.activation(t, act), y.numpy(), rtol=1e-11, atol=1e-15), act
        step = np.diff(L.activation(t, act)) / np.diff(t)
        assert (np.abs(step) <= L.slope(np.maximum(np.abs(t[1:]), np.abs(t[:-1])), act) + 1e-9).all(), act


def test_fp32_forms_stay_within_their_bound():
    """The library's formulas evaluated in numpy's fp32 (with its exact exp2 and division)."""
    f = np.float32
    t = np.concatenate([np.linspace(-30, 30, 20001), np.logspace(-8, 1, 500), -np.logspace(-8, 1, 500)]).astype(f)
    with np.errstate(over="ignore"):
        for act, c1, c3 in (("silu", -1.44269504, 0.0), ("gelu_tanh", -2.30220820, -0.102943240)):
            p = t * (t * t * f(c3) + f(c1))
            y = t / (f(1) + np.exp2(p))
            assert (np.abs(y - L.activation(t, act)) <= L.activation_error(t, act)).all(), act


def test_dequantised_epilogue_by_hand():
    acc = np.array([[3, -2, 5, 7]], np.int32)
    t = L.dequantised(acc, np.array([0.5], np.float32), np.array([1, 2, 4, 0.25], np.float32),
                      np.array([0.25, 1, -12, 0], np.float16))
    assert t.tolist() == [[1.75, -1.0, -2.0, 0.875]]
    assert L.exact(t, "relu", True).tolist() == [[-3.5, 0.0]]
    assert L.exact(t, "relu2", False, np.ones((1, 4), np.float16)).tolist() == [[4.0625, 1.0, 1.0, 1.765625]]
    y, e = L.epilogue(t, "relu", True)
    assert y.tolist() == [[-3.5, 0.0]] and (e < 0.01).all()


def test_pairs():
    W = np.arange(32)[:, None] * np.ones((1, 3))
    assert L.paired_rows(W)[:, 0].tolist() == (list(range(0, 8)) + list(range(16, 24)) + list(range(8, 16))
                                                + list(range(24, 32)))


@pytest.mark.parametrize("center", [False, True])
def test_norm(center):
    rng = np.random.default_rng(3)
    h, y = rng.normal(0, 2, (6, 40)).astype(np.float32), rng.normal(1, 1, (6, 40)).astype(np.float16)
    w, wp = rng.normal(1, .2, 40).astype(np.float16), rng.normal(1, .2, 40).astype(np.float16)
    gate, scale, shift = (rng.normal(0, .5, (3, 40)).astype(np.float16) for _ in range(3))
    seq = np.array([0, 2, 1, 1, 7, -1])
    n, h2 = L.norm(h, y, w, wp, gate, 0.5, scale, shift, seq, 1e-5, center)
    T = lambda a: torch.from_numpy(np.asarray(a, np.float64))  # noqa: E731
    row = T(np.clip(seq, 0, 2)).long()
    unit = (lambda x: F.layer_norm(x, (40,), eps=1e-5)) if center else (  # noqa: E731
        lambda x: x / (x.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt())
    hh = T(h) + 0.5 * T(gate)[row] * unit(T(y)) * T(wp)
    nn = unit(hh) * T(w) * (1 + T(scale)[row]) + T(shift)[row]
    assert np.allclose(h2, hh.numpy(), rtol=1e-5, atol=1e-6) and np.allclose(n, nn.numpy(), rtol=1e-5, atol=1e-5)


def test_gate_and_quantiser():
    n = np.arange(-32, 32, dtype=np.float32)[None].repeat(2, 0)
    g = L.gated(n, np.array([0, 1]), 3, 2)
    assert (g[0, 59:62] == 0).all() and (g[0, 62:] == n[0, 62:]).all() and (g[1, 62:] == 0).all()
    n[1, 5] = np.inf
    q, s = L.quantise(n, 8)
    assert s[0] == np.float32(32) / np.float32(127) and np.isnan(s[1]) and (q[1] == 0).all()
