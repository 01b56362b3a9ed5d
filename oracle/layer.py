"""Reference for what stands between a layer's quantised products: fused epilogues and
norms with the residual stream.  TEST INFRASTRUCTURE ONLY.

Only the tests may import this module.  It shares no code with the HIP library.

Where the interface fixes single fp32 operations (dequantisation, bias, gate,
residual, the norm behind its statistics) they are done one numpy fp32 operation
each, so results are compared bit for bit; activations are in fp64, with a bound
on what the library's fp32 evaluation may differ by.
"""
from __future__ import annotations

import math

import numpy as np
from scipy.special import ndtr

from . import oracle as O

F32 = np.float32
U = 2.0 ** -24                         # half a step of fp32


def paired_rows(W):
    """Rows [gates, ups] as blocks of 8 gates and their 8 ups."""
    half = len(W) // 2
    out = []
    for g in range(half // 8):
        out += [W[8 * g:8 * g + 8], W[half + 8 * g:half + 8 * g + 8]]
    return np.concatenate(out) if out else W


# ---- activations -----------------------------------------------------------------------------------------

EXACT = ("none", "relu", "relu2")


def activation(t, act):
    """fp64 value of act at fp32 t."""
    t = np.asarray(t, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "none":
            return t.copy()
        if act in ("relu", "relu2"):
            r = np.where(t < 0, 0.0, t)
            return r if act == "relu" else r * r
        if act == "silu":
            return t / (1 + np.exp(-t))
        if act == "gelu":
            return t * ndtr(t)
        assert act == "gelu_tanh"
        return t / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)))


def activation_error(t, act):
    """How far an fp32 evaluation of act at t may be from activation(t), by its steps.

    silu and gelu_tanh are x / (1 + exp2(p)): an error d of p moves the quotient by at most
    d ln 2 of itself; p has 2 (silu) or 5 roundings of 2^-24 of its size, constants included;
    exp2 and the reciprocal are good to one step (2^-23), the sum and the product round.
    gelu is x Phi(x), Phi by erfc(z) = q exp2(P(q) - z^2 log2 e): the fit 1.1e-7; the exponent
    t^2 / 2 with three roundings, P with the roundings of eight steps on partial sums below 4 and of
    its coefficients (11 in sum), 40 units in all with exp2, reciprocal and product.  Below 2^-100
    a result may be flushed to zero."""
    t = np.asarray(t, np.float64)
    y = np.abs(activation(t, act))
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "none" or act == "relu":
            return np.zeros_like(y)
        if act == "relu2":
            return y * U
        if act == "silu":
            rel = 2 * np.abs(t) * U + 6 * U
        elif act == "gelu":
            rel = (1.5 * t * t + 40) * U + 1.1e-7
        else:
            rel = 5 * np.abs(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)) * U + 6 * U
        return y * rel + 2.0 ** -100


def slope(t, act):
    """An upper bound of |d act / dt| at and around t."""
    if act == "relu2":
        return 2 * np.abs(t) + 1e-3
    return np.full_like(np.asarray(t, np.float64), 1.0 if act in ("none", "relu") else 1.13)


# ---- products --------------------------------------------------------------------------------------------

def dequantised(acc, s_a, s_w, bias=None):
    """t in fp32 from exact int32 sums."""
    t = (acc.astype(F32) * s_a[:, None].astype(F32)) * s_w.astype(F32)
    return t if bias is None else t + bias.astype(F32)


def epilogue(t, act="none", glu=False, residual=None, t_error=None, dtype=np.float16):
    """(Y before its rounding to dtype in fp64, bound of the library's distance from it, that
    rounding included).  t fp32 (or fp64 with t_error, what it may be off by).  Where no
    activation is approximated and t is exact, exact(...) gives the bits."""
    t = np.asarray(t, np.float64)
    err = np.zeros_like(t) if t_error is None else t_error
    half = t.shape[1] // 2
    a, a_err = (t[:, :half], err[:, :half]) if glu else (t, err)
    y = activation(a, act)
    e = activation_error(a, act) + a_err * slope(np.abs(a) + a_err, act)
    if glu:
        up, up_err = t[:, half:], err[:, half:]
        with np.errstate(invalid="ignore", over="ignore"):
            e = e * (np.abs(up) + up_err) + np.abs(y) * up_err
            y = y * up
            e = e + (np.abs(y) + e) * U
    if residual is not None:
        y = y + residual.astype(np.float64)
        e = e + (np.abs(y) + e) * U
    step, least = (2.0 ** -11, 2.0 ** -25) if dtype == np.float16 else (U, 2.0 ** -150)
    return y, e + (np.abs(y) + e) * step + least


def exact(t, act="none", glu=False, residual=None, dtype=np.float16):
    """Y's bits from t's, for activations that fp32 arithmetic gives exactly."""
    assert act in EXACT
    half = t.shape[1] // 2
    a = t[:, :half] if glu else t
    with np.errstate(over="ignore", invalid="ignore"):
        y = a if act == "none" else np.where(a < 0, F32(0), a)
        if act == "relu2":
            y = y * y
        if glu:
            y = y * t[:, half:]
        if residual is not None:
            y = y + residual.astype(F32)
        return y.astype(dtype)


# ---- norms -----------------------------------------------------------------------------------------------

def _mean(values):
    return math.fsum(values) / len(values) if np.all(np.isfinite(values)) else float(np.sum(values))


def statistics(x, eps, center):
    """fp32 mean (0 unless center) and 1 / sqrt(mean square + eps) of each row."""
    mean, rate = np.zeros((len(x), 1), F32), np.zeros((len(x), 1), F32)
    for i, row in enumerate(np.asarray(x, np.float64)):
        m = _mean(row) if center else 0.0
        mean[i] = m
        rate[i] = 1.0 / math.sqrt(_mean((row - m) ** 2) + eps)
    return mean, rate


def norm(h, y=None, weight=None, post_weight=None, gate=None, alpha=1.0, scale=None, shift=None, seq=None, eps=1e-6,
         center=False):
    """(n fp32, h' of h's type), one fp32 operation at a time."""
    with np.errstate(over="ignore", invalid="ignore"):
        pick = (lambda r: r.astype(F32)[np.clip(seq, 0, len(r) - 1)] if seq is not None else r.astype(F32)[:1])

        def unit(x):
            m, r = statistics(x, eps, center)
            x = x.astype(F32)
            return (x - m if center else x) * r
        if y is not None:
            u = y.astype(F32)
            if post_weight is not None:
                u = unit(y) * post_weight.astype(F32)
            if gate is not None:
                u = u * pick(gate)
            h = (h.astype(F32) + u * F32(alpha)).astype(h.dtype)
        n = unit(h)
        if weight is not None:
            n = n * weight.astype(F32)
        if scale is not None:
            n = n * (F32(1) + pick(scale))
        if shift is not None:
            n = n + pick(shift)
        return n, h


def gated(n, state, dm, du):
    """Rows with the columns of the other state's band set to zero."""
    if state is None:
        return n
    out = n.copy()
    K = n.shape[1]
    for i, s in enumerate(state):
        if s:
            out[i, K - du:] = 0
        else:
            out[i, K - dm - du:K - du] = 0
    return out


def quantise(n, bits):
    """Codes (packed for 4 bits) and scales; a row that is not finite has scale NaN and zero codes."""
    bad = ~np.isfinite(n).all(1)
    q, s = (O.quant_rows if bits == 4 else O.quant_rows_q8)(np.where(bad[:, None], F32(0), n).astype(F32))[:2]
    s = s.copy()
    s[bad] = np.nan
    return q, s


def quantise_gated(n, state, dm, du, bits):
    """The same of gated rows; what a state drops counts for whether a row is finite."""
    q, s = quantise(gated(n, state, dm, du), bits)
    bad = ~np.isfinite(n).all(1)
    q, s = q.copy(), s.copy()
    q[bad], s[bad] = 0, np.nan
    return q, s
