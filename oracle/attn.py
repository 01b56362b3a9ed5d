"""Reference for rotary positions, the paged 8-bit cache, attention over it and
weight-only products.  TEST INFRASTRUCTURE ONLY.

Only the tests may import this module.  It shares no code with the HIP library:
plain loops over sequences, pages and heads, in fp64 except where the interface
fixes fp32 arithmetic (scales and codes of unrotated values).
"""
from __future__ import annotations

import math

import numpy as np


# ---- rotary positions ------------------------------------------------------------------------------------

def frequencies(rot, base, scaling="none", factor=1.0, original=0.0, beta_fast=32.0, beta_slow=1.0):
    out = []
    for j in range(rot // 2):
        b = base
        if scaling == "ntk" and rot > 2:
            b = base * factor ** (rot / (rot - 2))
        f = b ** (-2.0 * j / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "yarn":
            turns = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)))
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return np.array(out)


def pair_index(rot, layout):
    j = np.arange(rot // 2)
    return (j, j + rot // 2) if layout == "half" else (2 * j, 2 * j + 1)


def rope(x, pos, freq, layout="half", amplitude=1.0, transpose=False):
    """[T, H, D] in fp64; pos [T]."""
    y = np.array(x, np.float64)
    a, b = pair_index(2 * len(freq), layout)
    ang = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang) * (-1 if transpose else 1)
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a] = u * c - v * s
    y[..., b] = v * c + u * s
    return y


# ---- the cache -------------------------------------------------------------------------------------------

class Cache:
    def __init__(self, pages, heads, dim, page):
        self.k = np.zeros((pages, heads, page, dim), np.int8)
        self.v = np.zeros((pages, heads, dim, page), np.int8)
        self.ks = np.zeros((pages, heads), np.float32)
        self.vs = np.zeros((pages, heads), np.float32)
        self.pages, self.heads, self.dim, self.page = pages, heads, dim, page

    def copy(self):
        c = Cache(self.pages, self.heads, self.dim, self.page)
        c.k, c.v, c.ks, c.vs = self.k.copy(), self.v.copy(), self.ks.copy(), self.vs.copy()
        return c


def _quantised(x, old, fresh):
    """fp32 scale and codes of x [tokens, D] against a page's scale `old`; NaN and zero codes if one is not finite."""
    s = np.float32(np.abs(x).max(initial=0.0).astype(np.float32) / np.float32(127))
    if not fresh:
        s = np.maximum(np.float32(old), s)             # NaN if one is
    if not np.isfinite(s):
        s = np.float32(np.nan)
    if not s > 0:
        return s, np.zeros(x.shape, np.int8)
    q = np.rint((x.astype(np.float32) / s).astype(np.float32))
    return s, np.clip(q, -128, 127).astype(np.int8)


def spans(cu, lens, table, page, pages):
    """(page id, first slot, end slot, first row) of each page that a batch writes."""
    out = []
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        p = int(lens[b]) - n
        t = int(cu[b])
        if p < 0:
            t, p = t - p, 0
        while p < lens[b] and t < cu[b + 1]:
            end = min(int(lens[b]), (p // page + 1) * page)
            pid = int(table[b, p // page])
            if 0 <= pid < pages:
                out.append((pid, p % page, p % page + end - p, t))
            t, p = t + end - p, end
    return out


def positions(cu, lens, T):
    pos = np.full(T, -1, np.int64)
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        pos[cu[b]:cu[b + 1]] = int(lens[b]) - n + np.arange(n)
    return pos


def append(cache, K, V, cu, lens, table):
    """K, V [T, heads, D] (K already rotated) into the cache, in place."""
    for pid, s0, s1, t in spans(cu, lens, table, cache.page, cache.pages):
        for h in range(cache.heads):
            for x, scales, codes in ((K, cache.ks, cache.k[pid, h]), (V, cache.vs, cache.v[pid, h].T)):
                old = scales[pid, h]
                s, q = _quantised(np.asarray(x[t:t + s1 - s0, h]), old, s0 == 0)
                if s0 and s > old:
                    ratio = np.float32(old / s)
                    codes[:s0] = np.rint(codes[:s0].astype(np.float32) * ratio).astype(np.int8)
                codes[s0:s1] = q
                scales[pid, h] = s


def values(cache, pids):
    """Pages as fp64 values: K, V [n, heads, page, D]; zeros where there is no page."""
    ok = (pids >= 0) & (pids < cache.pages)
    i = np.where(ok, pids, 0)
    k = cache.k[i].astype(np.float64) * cache.ks[i][..., None, None]
    v = cache.v[i].transpose(0, 1, 3, 2).astype(np.float64) * cache.vs[i][..., None, None]
    return k * ok[:, None, None, None], v * ok[:, None, None, None]


# ---- attention -------------------------------------------------------------------------------------------

def attention(q, cache, cu, lens, table, causal=True, window=0, scale=None):
    """Per row: out, lse, and what the error bounds need: sum p |v|, the largest |v scale|, the softmax's sum
    relative to its largest term, the number of terms and the largest sum |q c| of a logit."""
    T, Hq, D = q.shape
    G = Hq // cache.heads
    scale = D ** -0.5 if scale is None else scale
    out = np.full((T, Hq, D), np.nan)
    lse = np.full((T, Hq), np.nan)
    spread, vmax, total, terms, mass = (np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.ones((T, Hq)),
                                        np.zeros((T, Hq)), np.zeros((T, Hq)))
    for b in range(len(lens)):
        n, L = int(cu[b + 1] - cu[b]), int(lens[b])
        pids = np.asarray(table[b, :-(-L // cache.page)], np.int64)
        k, v = values(cache, pids)
        there = np.repeat((pids >= 0) & (pids < cache.pages), cache.page)[:L]
        k = k.transpose(1, 0, 2, 3).reshape(cache.heads, -1, D)[:, :L]
        v = v.transpose(1, 0, 2, 3).reshape(cache.heads, -1, D)[:, :L]
        big = cache.vs[np.where((pids >= 0) & (pids < cache.pages), pids, 0)].max(0, initial=0.0) if len(pids) else None
        for i in range(n):
            p, t = L - n + i, int(cu[b]) + i
            j = np.arange(L)
            see = there.copy()
            if causal:
                see &= j <= p
            if window:
                see &= j > p - window
            for h in range(Hq):
                kk, vv = k[h // G][see], v[h // G][see]
                if not len(kk):
                    out[t, h], lse[t, h] = 0.0, -np.inf
                    continue
                x = kk @ q[t, h].astype(np.float64) * scale
                m = x.max()
                w = np.exp(x - m)
                lse[t, h] = m + np.log(w.sum())
                total[t, h], terms[t, h] = w.sum(), len(w)
                w /= w.sum()
                out[t, h] = w @ vv
                spread[t, h] = w @ np.abs(vv)
                vmax[t, h] = big[h // G]
                mass[t, h] = (np.abs(kk) @ np.abs(q[t, h].astype(np.float64))).max() * abs(scale)
    return out, lse, dict(spread=spread, vmax=vmax, total=total, terms=terms, mass=mass)


def attention_bounds(out, lse, e, D, floor=2.0 ** -36):
    """How far fp32 sums and logits, fp16 weights and one fp16 rounding may be from fp64.

    A logit sums D products in fp32 (each addition 2^-24 of the sum of magnitudes) and is scaled twice and
    subtracted from the reference (3 roundings); 2^x of fp32 adds 2^-22 relative.  A weight times its value scale is
    rounded to fp16: half a step, 2^-11 relative or, below fp16's normal range, 2^-25 where the row's largest is at
    2^11 or more: `floor` of the largest value scale, for codes up to 128; the softmax's sum is at least its largest
    term, 1.  Both sums over the terms are in fp32."""
    logit = (D + 6) * 2.0 ** -24 * e["mass"] + 2.0 ** -21
    rel = 2.0 ** -11 + 2 * logit + e["terms"] * 2.0 ** -23 + 2.0 ** -20
    b_out = (2.0 ** -11 * np.abs(out) + 2.0 ** -25 + rel[..., None] * e["spread"]
             + (e["terms"] * floor * 128 * e["vmax"] / e["total"])[..., None])
    b_lse = logit + e["terms"] * 2.0 ** -24 + 2.0 ** -20 + 4 * 2.0 ** -24 * np.abs(np.where(np.isfinite(lse), lse, 0))
    return b_out, b_lse


# ---- weight-only products --------------------------------------------------------------------------------

def quantize_group(W, group):
    """W [N, K] fp16 -> codes [N, K] and fp16 scales [K / group, N]."""
    N, K = W.shape
    x = np.asarray(W, np.float32).reshape(N, K // group, group)
    s = (np.abs(x).max(-1) / np.float32(7)).astype(np.float32).astype(np.float16)
    sf = s.astype(np.float32)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where((sf > 0) & np.isfinite(sf), np.clip(np.rint(x / sf), -8, 7), 0)
    return q.reshape(N, K).astype(np.int64), np.ascontiguousarray(s.T)


def w4a16(X, codes, s, group):
    """Y in fp64 and sum |x q s| of each output."""
    w = codes.astype(np.float64) * np.repeat(s.astype(np.float64).T, group, axis=1)
    x = X.astype(np.float64)
    return x @ w.T, np.abs(x) @ np.abs(w).T
