"""STaR-Quant W4A4 hot path on MI355X (gfx950): thin torch binding of libstarquant.

Every function here only checks and marshals arguments (device pointers, sizes,
the current HIP stream) and calls the C ABI declared in include/starquant.h;
all arithmetic runs in the library's HIP kernels.  torch provides device memory
and streams.  Outputs and workspaces are allocated with torch when not given.

    Aq, s_a = sgat_quant_act(X, state, P)            # Eq. 11 + per-token int4
    Wq, s_w = sgat_prepare_weights(W, P)             # Eq. 12, offline
    Y = w4a4_gemm(Aq, s_a, Wq, s_w)                  # Eq. 13
    Zc = tac_apply(Z, tac_M, tac_d, g)               # Eq. 17

Between the projections, attention over a paged 8-bit cache:

    cache = kv_cache(pages, heads, dim)
    freq = rope_frequencies(dim, 1e6)
    q = kv_append(cache, k, v, cu, lens, table, freq=freq, q=q)
    Z = attn_kv8(q, cache, cu, lens, table)

Between the products, the residual stream, norms and activations:

    Aq, s_a, h = norm_quant(h, y, weight=w, state=state)
    y = w4a4_linear(Aq, s_a, Wf, s_w, act="silu", glu=True)
    h = w4a4_linear(*sgat_quant_act(y, state), Wf2, s_w2, residual=h)
"""
from __future__ import annotations

import functools
import math
from typing import NamedTuple, Optional, Tuple

import torch

from ._lib import EPILOGUE, NORM_ARGS, KVCacheStruct, SQ_OK, StarQuantError, check, lib  # noqa: F401

__all__ = ["sgat_prepare_weights", "sgat_transform", "sgat_quantize", "sgat_quant_act", "w4a4_gemm", "tac_apply",
           "tac_default_block", "default_band", "quant_act_workspace_bytes", "gemm_workspace_bytes",
           "prepare_weights_workspace_bytes", "StarQuantError", "lib",
           "sgat_prepare_weights_w8", "sgat_quantize_w8", "sgat_quant_act_w8", "w8a8_gemm",
           "tac_calibrate", "tac_calibrate_workspace_bytes", "sgat_split_basis", "sgat_transform_fast",
           "fp6_row_bytes", "codes_to_fp6", "w4a4_gemm_fp6",
           "frag_weight_bytes", "weights_to_frag", "w4a4_gemm_frag", "w8a8_gemm_frag",
           "rope_frequencies", "rope_amplitude", "rope", "KVCache", "kv_cache", "kv_append", "kv_read", "attn_kv8",
           "attn_kv8_workspace_bytes", "quantize_weights_group", "w4a16_gemm_frag",
           "w4a4_linear", "w8a8_linear", "w4a16_linear", "norm", "norm_quant"]


def _on_stream(fn):
    """Runs a binding call with `stream` (when given) as torch's current stream,
    so that every tensor the call allocates (outputs, workspaces) belongs to the
    stream its kernels run on and the caching allocator cannot hand that memory
    to other work while they use it.  A raw HIP stream handle is wrapped as an
    external stream."""
    @functools.wraps(fn)
    def wrapper(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))
        with torch.cuda.stream(s):
            return fn(*args, stream=s, **kw)
    return wrapper


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The current stream's handle without the Stream object that
# torch.cuda.current_stream() builds (0.1 against 2.7 us of host time, in a call
# whose launch takes 3.4); the arguments were seen to be device tensors first, so
# the runtime is up.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _need(t: Optional[torch.Tensor], name: str, dtype, shape=None, optional=False):
    # what holds on every good call, in one test (0.2 us); the message otherwise
    if t is not None and t.is_cuda and t.dtype is dtype and t.is_contiguous() and (shape is None or t.shape == shape):
        return
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _ws(nbytes: int, ws: Optional[torch.Tensor], device) -> Tuple[Optional[torch.Tensor], int]:
    if nbytes == 0:
        return ws, (ws.numel() if ws is not None else 0)
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.numel() * ws.element_size()


def tac_default_block(C: int) -> int:
    return int(lib().sq_tac_default_block(int(C)))


def default_band(K: int) -> Tuple[int, int]:
    """d_m = d_u = K/32 (App. B default subspace allocation)."""
    return K // 32, K // 32


def quant_act_workspace_bytes(M: int, K: int, has_P: bool, has_tac: bool) -> int:
    return int(lib().sq_quant_act_workspace_bytes(M, K, int(has_P), int(has_tac)))


_quant_workspace_bytes = functools.lru_cache(maxsize=4096)(quant_act_workspace_bytes)      # of sizes alone


def prepare_weights_workspace_bytes(N: int, K: int, has_P: bool) -> int:
    return int(lib().sq_prepare_weights_workspace_bytes(N, K, int(has_P)))


def gemm_workspace_bytes(M: int, N: int, K: int, bits: int = 4) -> int:
    f = lib().sq_gemm_w8_workspace_bytes if bits == 8 else lib().sq_gemm_workspace_bytes
    return int(f(M, N, K))


def _codes_spec(bits: int, K: int):
    """(dtype, row width) of a code tensor: packed int4 uint8 [K/2] or int8 [K]."""
    return (torch.int8, K) if bits == 8 else (torch.uint8, K // 2)


@_on_stream
def sgat_prepare_weights(W: torch.Tensor, P: Optional[torch.Tensor] = None, *, Wq=None, s_w=None, ws=None,
                         stream=None, bits: int = 4):
    """W~ = Q_w(P^T W^T) as rows of W P: returns (Wq, s_w [N] fp32); Wq is [N][K/2]
    packed int4 (bits=4) or [N][K] int8 (bits=8, App. D)."""
    N, K = W.shape
    dt, kw = _codes_spec(bits, K)
    _need(W, "W", torch.float16)
    _need(P, "P", torch.float32, (K, K), optional=True)
    if Wq is None:
        Wq = torch.empty((N, kw), dtype=dt, device=W.device)
    if s_w is None:
        s_w = torch.empty((N,), dtype=torch.float32, device=W.device)
    _need(Wq, "Wq", dt, (N, kw))
    _need(s_w, "s_w", torch.float32, (N,))
    ws, wsb = _ws(prepare_weights_workspace_bytes(N, K, P is not None), ws, W.device)
    f = lib().sgat_prepare_weights_w8 if bits == 8 else lib().sgat_prepare_weights
    check(f(_ptr(W), _ptr(P), N, K, _ptr(Wq), _ptr(s_w), _ptr(ws), wsb, _stream(stream)))
    return Wq, s_w


def sgat_prepare_weights_w8(W, P=None, **kw):
    return sgat_prepare_weights(W, P, bits=8, **kw)


@_on_stream
def sgat_transform(X: torch.Tensor, state: Optional[torch.Tensor], P: Optional[torch.Tensor],
                   d_m: Optional[int] = None, d_u: Optional[int] = None, *, out=None, stream=None):
    """x'_i = x_i P G_{s_i} (Eq. 11), fp32 [M][K]."""
    M, K = X.shape
    dm0, du0 = default_band(K)
    d_m = dm0 if d_m is None else d_m
    d_u = du0 if d_u is None else d_u
    _need(X, "X", torch.float16)
    _need(state, "state", torch.uint8, (M,), optional=True)
    _need(P, "P", torch.float32, (K, K), optional=True)
    if out is None:
        out = torch.empty((M, K), dtype=torch.float32, device=X.device)
    _need(out, "out", torch.float32, (M, K))
    check(lib().sgat_transform(_ptr(X), _ptr(state), _ptr(P), M, K, d_m, d_u, _ptr(out), _stream(stream)))
    return out


@_on_stream
def sgat_quantize(Xp: torch.Tensor, *, Aq=None, s=None, stream=None, bits: int = 4):
    """Per-row symmetric quantisation of fp32 rows (Eq. 2, z = 0): returns (Aq, s [M] fp32)."""
    M, K = Xp.shape
    dt, kw = _codes_spec(bits, K)
    _need(Xp, "Xp", torch.float32)
    if Aq is None:
        Aq = torch.empty((M, kw), dtype=dt, device=Xp.device)
    if s is None:
        s = torch.empty((M,), dtype=torch.float32, device=Xp.device)
    _need(Aq, "Aq", dt, (M, kw))
    _need(s, "s", torch.float32, (M,))
    f = lib().sgat_quantize_w8 if bits == 8 else lib().sgat_quantize
    check(f(_ptr(Xp), M, K, _ptr(Aq), _ptr(s), _stream(stream)))
    return Aq, s


def sgat_quantize_w8(Xp, **kw):
    return sgat_quantize(Xp, bits=8, **kw)


@_on_stream
def sgat_quant_act(X: torch.Tensor, state: Optional[torch.Tensor], P: Optional[torch.Tensor] = None,
                   d_m: Optional[int] = None, d_u: Optional[int] = None, tac_M: Optional[torch.Tensor] = None,
                   tac_d: Optional[torch.Tensor] = None, g: int = 0, *, Aq=None, s_a=None, ws=None, stream=None,
                   bits: int = 4):
    """[TAC] -> x P G_s -> per-token codes: returns (Aq, s_a [M] fp32), Aq packed int4
    [M][K/2] uint8 (bits=4) or int8 [M][K] (bits=8)."""
    M, K = X.shape
    dt, kw = _codes_spec(bits, K)
    dm0, du0 = default_band(K)
    d_m = dm0 if d_m is None else d_m
    d_u = du0 if d_u is None else d_u
    _need(X, "X", torch.float16)
    _need(state, "state", torch.uint8, (M,), optional=True)
    _need(P, "P", torch.float32, (K, K), optional=True)
    if tac_M is not None:
        _need(tac_M, "tac_M", torch.float16, (K // g, g, g))
        _need(tac_d, "tac_d", torch.float16, (K,))
    if Aq is None:
        Aq = X.new_empty((M, kw), dtype=dt)
    else:
        _need(Aq, "Aq", dt, (M, kw))
    if s_a is None:
        s_a = X.new_empty((M,), dtype=torch.float32)
    else:
        _need(s_a, "s_a", torch.float32, (M,))
    ws, wsb = _ws(_quant_workspace_bytes(M, K, P is not None, tac_M is not None), ws, X.device)
    f = lib().sgat_quant_act_w8 if bits == 8 else lib().sgat_quant_act
    check(f(_ptr(X), _ptr(state), _ptr(P), M, K, d_m, d_u, _ptr(tac_M), _ptr(tac_d), g,
            _ptr(Aq), _ptr(s_a), _ptr(ws), wsb, _stream(stream)))
    return Aq, s_a


def sgat_quant_act_w8(X, state, P=None, d_m=None, d_u=None, tac_M=None, tac_d=None, g=0, **kw):
    return sgat_quant_act(X, state, P, d_m, d_u, tac_M, tac_d, g, bits=8, **kw)


@_on_stream
def w4a4_gemm(Aq: torch.Tensor, s_a: torch.Tensor, Wq: torch.Tensor, s_w: torch.Tensor, *, Y=None, acc=None,
              want_Y: bool = True, want_acc: bool = False, ws=None, stream=None, bits: int = 4):
    """Y = fp16((acc * s_a) * s_w) with acc = Aq . Wq^T exact (Eq. 13).  Returns Y, or (Y, acc).
    bits=8 takes int8 codes (App. D)."""
    M, Kc = Aq.shape
    N = Wq.shape[0]
    dt = torch.int8 if bits == 8 else torch.uint8
    K = Kc if bits == 8 else 2 * Kc
    _need(Aq, "Aq", dt)
    _need(Wq, "Wq", dt, (N, Kc))
    _need(s_a, "s_a", torch.float32, (M,))
    _need(s_w, "s_w", torch.float32, (N,))
    if Y is None and want_Y:
        Y = torch.empty((M, N), dtype=torch.float16, device=Aq.device)
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=Aq.device)
    _need(Y, "Y", torch.float16, (M, N), optional=True)
    _need(acc, "acc", torch.int32, (M, N), optional=True)
    ws, wsb = _ws(gemm_workspace_bytes(M, N, K, bits), ws, Aq.device)
    f = lib().w8a8_gemm if bits == 8 else lib().w4a4_gemm
    check(f(_ptr(Aq), _ptr(s_a), _ptr(Wq), _ptr(s_w), M, N, K, _ptr(Y), _ptr(acc), _ptr(ws), wsb, _stream(stream)))
    return (Y, acc) if want_acc else Y


def w8a8_gemm(Aq, s_a, Wq, s_w, **kw):
    return w4a4_gemm(Aq, s_a, Wq, s_w, bits=8, **kw)


def fp6_row_bytes(K: int) -> int:
    """Bytes per row of an FP6 operand of K codes (96 per block of 128)."""
    n = int(lib().sq_fp6_row_bytes(K))
    if n == 0:
        raise ValueError(f"K={K}: need 64 <= K <= 131072 and K % 64 == 0")
    return n


@_on_stream
def codes_to_fp6(codes: torch.Tensor, *, out=None, stream=None):
    """Packed int4 codes [R, K/2] -> the FP6 (e3m2) operand layout [R, fp6_row_bytes(K)]."""
    R, Kh = codes.shape
    K = 2 * Kh
    _need(codes, "codes", torch.uint8)
    rb = fp6_row_bytes(K)
    if out is None:
        out = torch.empty((R, rb), dtype=torch.uint8, device=codes.device)
    _need(out, "out", torch.uint8, (R, rb))
    check(lib().sq_codes_to_fp6(_ptr(codes), R, K, _ptr(out), _stream(stream)))
    return out


@_on_stream
def w4a4_gemm_fp6(A6: torch.Tensor, s_a: torch.Tensor, W6: torch.Tensor, s_w: torch.Tensor, K: int, *, Y=None,
                  acc=None, want_Y: bool = True, want_acc: bool = False, stream=None):
    """The W4A4 GEMM (Eq. 13) on FP6 operands (codes_to_fp6 layout) and the FP6
    matrix cores; bit-identical to w4a4_gemm.  Returns Y, or (Y, acc)."""
    M, N = A6.shape[0], W6.shape[0]
    rb = fp6_row_bytes(K)
    _need(A6, "A6", torch.uint8, (M, rb))
    _need(W6, "W6", torch.uint8, (N, rb))
    _need(s_a, "s_a", torch.float32, (M,))
    _need(s_w, "s_w", torch.float32, (N,))
    if Y is None and want_Y:
        Y = torch.empty((M, N), dtype=torch.float16, device=A6.device)
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=A6.device)
    _need(Y, "Y", torch.float16, (M, N), optional=True)
    _need(acc, "acc", torch.int32, (M, N), optional=True)
    check(lib().w4a4_gemm_fp6(_ptr(A6), _ptr(s_a), _ptr(W6), _ptr(s_w), M, N, K, _ptr(Y), _ptr(acc),
                              _stream(stream)))
    return (Y, acc) if want_acc else Y


def frag_weight_bytes(N: int, K: int, bits: int = 4) -> int:
    """Bytes of the fragment-ordered weights of an N x K code matrix (1 KB per
    16 rows and k step of 64 bytes: 128 int4 or 64 int8 codes)."""
    n = int(lib().sq_frag_weight_w8_bytes(N, K) if bits == 8 else lib().sq_frag_weight_bytes(N, K))
    if n == 0 and N > 0:
        kmax = 65536 if bits == 8 else 131072
        raise ValueError(f"K={K}: need 64 <= K <= {kmax} and K % 64 == 0")
    return n


@functools.lru_cache(maxsize=4096)
def _frag_shape(N: int, K: int, bits: int):
    step = 64 if bits == 8 else 128
    return ((K + step - 1) // step, (N + 15) // 16, 1024)


@_on_stream
def weights_to_frag(Wq: torch.Tensor, *, glu: bool = False, out=None, stream=None):
    """Code matrix -> fragment order [k steps, ceil(N/16), 1024] (uint8): packed
    int4 weights [N, K/2] (uint8, 128 codes a k step) or int8 weights [N, K]
    (int8, 64 codes a k step).  glu=True: rows are N/2 gates and then their ups,
    stored in alternating blocks of 8 for the gated *_linear calls."""
    N, Kc = Wq.shape
    bits = 8 if Wq.dtype == torch.int8 else 4
    K = Kc if bits == 8 else 2 * Kc
    _need(Wq, "Wq", torch.int8 if bits == 8 else torch.uint8)
    shape = _frag_shape(N, K, bits)
    frag_weight_bytes(N, K, bits)
    if out is None:
        out = torch.empty(shape, dtype=torch.uint8, device=Wq.device)
    _need(out, "out", torch.uint8, shape)
    if glu:
        f = lib().sq_weights_to_frag_glu_w8 if bits == 8 else lib().sq_weights_to_frag_glu
    else:
        f = lib().sq_weights_to_frag_w8 if bits == 8 else lib().sq_weights_to_frag
    check(f(_ptr(Wq), N, K, _ptr(out), _stream(stream)))
    return out


@_on_stream
def w4a4_gemm_frag(Aq: torch.Tensor, s_a: torch.Tensor, Wf: torch.Tensor, s_w: torch.Tensor, *, Y=None, acc=None,
                   want_Y: bool = True, want_acc: bool = False, ws=None, stream=None, bits: int = 4):
    """w4a4_gemm (Eq. 13) with the weights in fragment order (weights_to_frag);
    N is s_w's length.  Bit-identical to w4a4_gemm.  bits=8 takes int8
    activation codes and the fragment order of int8 weights (App. D),
    bit-identical to w8a8_gemm.  Returns Y, or (Y, acc)."""
    M, Kc = Aq.shape
    N = s_w.shape[0]
    K = Kc if bits == 8 else 2 * Kc
    _need(Aq, "Aq", torch.int8 if bits == 8 else torch.uint8)
    _need(Wf, "Wf", torch.uint8, _frag_shape(N, K, bits))
    _need(s_a, "s_a", torch.float32, (M,))
    _need(s_w, "s_w", torch.float32, (N,))
    if Y is None and want_Y:
        Y = torch.empty((M, N), dtype=torch.float16, device=Aq.device)
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=Aq.device)
    _need(Y, "Y", torch.float16, (M, N), optional=True)
    _need(acc, "acc", torch.int32, (M, N), optional=True)
    ws, wsb = _ws(gemm_workspace_bytes(M, N, K, bits), ws, Aq.device)
    f = lib().w8a8_gemm_frag if bits == 8 else lib().w4a4_gemm_frag
    check(f(_ptr(Aq), _ptr(s_a), _ptr(Wf), _ptr(s_w), M, N, K, _ptr(Y), _ptr(acc), _ptr(ws), wsb, _stream(stream)))
    return (Y, acc) if want_acc else Y


def w8a8_gemm_frag(Aq, s_a, Wf, s_w, **kw):
    return w4a4_gemm_frag(Aq, s_a, Wf, s_w, bits=8, **kw)


@_on_stream
def tac_apply(Z: torch.Tensor, tac_M: torch.Tensor, tac_d: torch.Tensor, g: int, *, out=None, stream=None):
    """Z_b M_b^T + 1 d_b^T per block of g channels (Eq. 17), fp16 out."""
    M, C = Z.shape
    _need(Z, "Z", torch.float16)
    _need(tac_M, "tac_M", torch.float16, (C // g, g, g))
    _need(tac_d, "tac_d", torch.float16, (C,))
    if out is None:
        out = torch.empty_like(Z)
    _need(out, "out", torch.float16, (M, C))
    check(lib().tac_apply(_ptr(Z), _ptr(tac_M), _ptr(tac_d), M, C, g, _ptr(out), _stream(stream)))
    return out


TAC_RHO, TAC_EPS, TAC_ETA, TAC_ALPHA = 3e-4, 1e-8, 0.15, 0.55   # App. C defaults


def tac_calibrate_workspace_bytes(N: int, C: int, g: int) -> int:
    return int(lib().sq_tac_calibrate_workspace_bytes(N, C, g))


@_on_stream
def tac_calibrate(Z_fp: torch.Tensor, Z_q: torch.Tensor, g: int, *, rho: float = TAC_RHO, eps: float = TAC_EPS,
                  eta: float = TAC_ETA, alpha: float = TAC_ALPHA, want_fp64: bool = False, tac_M=None, tac_d=None,
                  ws=None, stream=None):
    """Closed-form TAC parameters (App. C) from paired full-precision / quantised
    attention outputs: (tac_M fp16 [C/g, g, g], tac_d fp16 [C]) and, with
    want_fp64, also the unrounded fp64 (M, d)."""
    N, C = Z_fp.shape
    _need(Z_fp, "Z_fp", torch.float16)
    _need(Z_q, "Z_q", torch.float16, (N, C))
    dev = Z_fp.device
    if tac_M is None:
        tac_M = torch.empty((C // g, g, g), dtype=torch.float16, device=dev)
    if tac_d is None:
        tac_d = torch.empty((C,), dtype=torch.float16, device=dev)
    _need(tac_M, "tac_M", torch.float16, (C // g, g, g))
    _need(tac_d, "tac_d", torch.float16, (C,))
    M64 = torch.empty((C // g, g, g), dtype=torch.float64, device=dev) if want_fp64 else None
    d64 = torch.empty((C,), dtype=torch.float64, device=dev) if want_fp64 else None
    ws, wsb = _ws(tac_calibrate_workspace_bytes(N, C, g), ws, dev)
    check(lib().tac_calibrate(_ptr(Z_fp), _ptr(Z_q), N, C, g, rho, eps, eta, alpha, _ptr(tac_M), _ptr(tac_d),
                              _ptr(M64), _ptr(d64), _ptr(ws), wsb, _stream(stream)))
    return (tac_M, tac_d, M64, d64) if want_fp64 else (tac_M, tac_d)


@_on_stream
def sgat_split_basis(P: torch.Tensor, *, out=None, stream=None):
    """fp16 hi / lo split of 2^14 P, transposed: Ps [K, 2K] for sgat_transform_fast."""
    K = P.shape[0]
    _need(P, "P", torch.float32, (K, K))
    if out is None:
        out = torch.empty((K, 2 * K), dtype=torch.float16, device=P.device)
    _need(out, "out", torch.float16, (K, 2 * K))
    check(lib().sgat_split_basis(_ptr(P), K, _ptr(out), _stream(stream)))
    return out


@_on_stream
def sgat_transform_fast(X: torch.Tensor, state: Optional[torch.Tensor], Ps: torch.Tensor,
                        d_m: Optional[int] = None, d_u: Optional[int] = None, *, out=None, stream=None):
    """x' = x P G_s on the fp16 matrix cores (within a stated bound of the exact
    product; not bit-identical to sgat_transform).  fp32 out."""
    M, K = X.shape
    _need(X, "X", torch.float16)
    _need(state, "state", torch.uint8, (M,), optional=True)
    _need(Ps, "Ps", torch.float16, (K, 2 * K))
    dm0, du0 = default_band(K)
    d_m = dm0 if d_m is None else d_m
    d_u = du0 if d_u is None else d_u
    if out is None:
        out = torch.empty((M, K), dtype=torch.float32, device=X.device)
    _need(out, "out", torch.float32, (M, K))
    check(lib().sgat_transform_fast(_ptr(X), _ptr(state), _ptr(Ps), M, K, d_m, d_u, _ptr(out), _stream(stream)))
    return out


ROPE_LAYOUTS = {"half": 0, "pairs": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


@functools.lru_cache(maxsize=None)
def _one_gpu() -> bool:
    return torch.cuda.device_count() == 1


def _run(fn, tensors, args, stream):
    """check(fn(*args, stream)) on the device that the tensors (None: not given) are all on,
    which need not be the current one."""
    if not _one_gpu():
        dev = tensors[0].get_device()
        for t in tensors:
            if t is not None and t.get_device() != dev:
                raise ValueError("the tensors are on different devices")
        if dev != torch.cuda.current_device():
            if stream is not None:
                raise ValueError("the stream is on another device than the tensors")
            with torch.cuda.device(dev):
                return check(fn(*args, _stream(None)))
    rc = fn(*args, _stream(stream))
    if rc != SQ_OK:
        check(rc)


def _choice(table: dict, key, name: str) -> int:
    if key not in table:
        raise ValueError(f"{name} must be one of {sorted(table)}, got {key!r}")
    return table[key]


@_on_stream
def rope_frequencies(rot: int, base: float, *, scaling: str = "none", factor: float = 1.0, original: float = 0.0,
                     beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda", out=None, stream=None):
    """Radians per position of each rotary pair, fp64 [rot / 2]: base^(-2 j / rot), scaled
    ("linear", "ntk" or "yarn") for contexts `factor` times the `original` length."""
    kind = _choice(ROPE_SCALINGS, scaling, "scaling")
    if out is None:
        out = torch.empty((max(0, rot // 2),), dtype=torch.float64, device=device)
    _need(out, "out", torch.float64, (rot // 2,))
    _run(lib().sq_rope_frequencies, (out,), (rot, base, kind, factor, original, beta_fast, beta_slow, _ptr(out)),
         stream)
    return out


def rope_amplitude(scaling: str, factor: float) -> float:
    """What a scaling multiplies cos and sin by: 0.1 ln(factor) + 1 for "yarn", else 1."""
    return float(lib().sq_rope_amplitude(_choice(ROPE_SCALINGS, scaling, "scaling"), factor))


def _heads(t: torch.Tensor, name: str, shape=None):
    """Checks a [T, H, D] fp16 device tensor, dense in D; returns its (token, head) strides."""
    # what holds on every good call, in one test; the message otherwise
    if t is not None and t.is_cuda and t.dtype is torch.float16 and (shape is None or t.shape == shape):
        s = t.stride()
        if len(s) == 3 and s[2] == 1:
            return s[:2]
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda or t.dtype is not torch.float16:
        raise ValueError(f"{name} must be a torch.float16 device tensor")
    if t.dim() != 3 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must have shape {tuple(shape) if shape else '[T, H, D]'}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be dense in its last dimension")


@_on_stream
def rope(X: torch.Tensor, freq: torch.Tensor, pos: Optional[torch.Tensor] = None, *, layout: str = "half",
         amplitude: float = 1.0, transpose: bool = False, out=None, stream=None):
    """Rotary positions on [T, H, D] heads (any strides of T and H that are multiples of 8):
    the first 2 len(freq) entries of each head turn by pos freq (pos [T] int32, default the
    token's index).  transpose=True applies the transposed map (the gradient).  out may be X."""
    T, H, D = X.shape
    xs = _heads(X, "X")
    _need(freq, "freq", torch.float64, (freq.numel(),))
    _need(pos, "pos", torch.int32, (T,), optional=True)
    if out is None:
        out, ys = X.new_empty((T, H, D)), (H * D, D)
    else:
        ys = _heads(out, "out", (T, H, D))
    _run(lib().sq_rope, (X, freq, pos, out),
         (_ptr(X), *xs, _ptr(pos), _ptr(freq), T, H, D, 2 * freq.numel(), _choice(ROPE_LAYOUTS, layout, "layout"),
          int(transpose), amplitude, _ptr(out), *ys), stream)
    return out


class KVCache(NamedTuple):
    """A paged 8-bit key / value cache: codes k [pages, heads, page, dim] and
    v [pages, heads, dim, page], fp32 scales [pages, heads]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def struct(self) -> KVCacheStruct:
        """The sq_kv_cache of this cache, its tensors checked."""
        if self.k.dim() != 4:
            raise ValueError(f"k must have shape [pages, heads, page, dim], got {tuple(self.k.shape)}")
        pages, heads, page, dim = self.k.shape
        _need(self.k, "k", torch.int8)
        _need(self.v, "v", torch.int8, (pages, heads, dim, page))
        _need(self.k_scale, "k_scale", torch.float32, (pages, heads))
        _need(self.v_scale, "v_scale", torch.float32, (pages, heads))
        return KVCacheStruct(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                             pages, page, heads, dim)


def kv_cache(pages: int, heads: int, dim: int, page: int = 64, device="cuda") -> KVCache:
    """An empty cache of `pages` pages of `page` tokens (zero codes and scales)."""
    return KVCache(torch.zeros((pages, heads, page, dim), dtype=torch.int8, device=device),
                   torch.zeros((pages, heads, dim, page), dtype=torch.int8, device=device),
                   torch.zeros((pages, heads), dtype=torch.float32, device=device),
                   torch.zeros((pages, heads), dtype=torch.float32, device=device))


def _batch(cu, lens, table):
    if lens is None or table is None or table.dim() != 2:
        raise ValueError("lens [B] and table [B, max_pages] are required")
    B, max_pages = table.shape
    _need(cu, "cu", torch.int32, (B + 1,))
    _need(lens, "lens", torch.int32, (B,))
    _need(table, "table", torch.int32)
    return B, max_pages


@_on_stream
def kv_append(cache: KVCache, K: torch.Tensor, V: torch.Tensor, cu: torch.Tensor, lens: torch.Tensor,
              table: torch.Tensor, *, freq: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
              layout: str = "half", amplitude: float = 1.0, q: Optional[torch.Tensor] = None, q_out=None, stream=None):
    """New tokens' keys (rotated when freq is given) and values [T, heads, dim] into the cache.
    Sequence b's tokens are rows cu[b] .. cu[b + 1] - 1 and the last of its lens[b] positions;
    position p lies in page table[b, p // page].  With q [T, Hq, dim] the queries are rotated
    too and returned (q_out may be q)."""
    c = cache.struct()
    B, max_pages = _batch(cu, lens, table)
    T = K.shape[0]
    ks = _heads(K, "K", (T, c.heads, c.dim))
    vs = _heads(V, "V", (T, c.heads, c.dim))
    _need(freq, "freq", torch.float64, None if freq is None else (freq.numel(),), optional=True)
    _need(pos, "pos", torch.int32, (T,), optional=True)
    qs = rs = (0, 0)
    Hq = 0
    if q is not None:
        if freq is None:
            raise ValueError("q needs freq")
        Hq = q.shape[1]
        qs = _heads(q, "q", (T, Hq, c.dim))
        if q_out is None:
            q_out, rs = q.new_empty((T, Hq, c.dim)), (Hq * c.dim, c.dim)
        else:
            rs = _heads(q_out, "q_out", (T, Hq, c.dim))
    else:
        q_out = None
    _run(lib().kv_append, (*cache, K, V, cu, lens, table, pos, freq, q, q_out),
         (c, _ptr(K), *ks, _ptr(V), *vs, _ptr(cu), _ptr(lens), _ptr(table), T, B, max_pages, _ptr(pos), _ptr(freq),
          0 if freq is None else 2 * freq.numel(), _choice(ROPE_LAYOUTS, layout, "layout"), amplitude, _ptr(q), *qs, Hq,
          _ptr(q_out), *rs), stream)
    return q_out


@_on_stream
def kv_read(cache: KVCache, pages: torch.Tensor, *, K=None, V=None, stream=None):
    """The listed pages (int32 [n]) as the values they hold: fp16 K and V [n, heads, page, dim]."""
    c = cache.struct()
    _need(pages, "pages", torch.int32, (pages.numel(),))
    shape = (pages.numel(), c.heads, c.page, c.dim)
    if K is None:
        K = pages.new_empty(shape, dtype=torch.float16)
    else:
        _need(K, "K", torch.float16, shape)
    if V is None:
        V = pages.new_empty(shape, dtype=torch.float16)
    else:
        _need(V, "V", torch.float16, shape)
    _run(lib().kv_read, (*cache, pages, K, V), (c, _ptr(pages), shape[0], _ptr(K), _ptr(V)), stream)
    return K, V


def attn_kv8_workspace_bytes(T: int, B: int, Hq: int, heads: int, dim: int, max_len: int) -> int:
    return int(lib().sq_attn_kv8_workspace_bytes(T, B, Hq, heads, dim, max_len))


@_on_stream
def attn_kv8(q: torch.Tensor, cache: KVCache, cu: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, *,
             causal: bool = True, window: int = 0, scale: Optional[float] = None, out=None, lse=None,
             want_lse: bool = False, ws=None, stream=None):
    """Attention of the queries [T, Hq, dim] over the cache; batch arguments as in kv_append,
    after which it is called.  scale defaults to dim^-0.5.  A row that sees no key gives zeros
    (lse -inf); rows of no sequence are left as they were.  Returns out [T, Hq, dim], or
    (out, lse [T, Hq] fp32)."""
    c = cache.struct()
    B, max_pages = _batch(cu, lens, table)
    T, Hq = q.shape[:2]
    qs = _heads(q, "q", (T, Hq, c.dim))
    if out is None:
        out = q.new_empty((T, Hq, c.dim))
    else:
        _need(out, "out", torch.float16, (T, Hq, c.dim))
    if lse is not None:
        _need(lse, "lse", torch.float32, (T, Hq))
    elif want_lse:
        lse = q.new_empty((T, Hq), dtype=torch.float32)
    if ws is not None:
        _need(ws, "ws", torch.uint8)
    ws, wsb = _ws(attn_kv8_workspace_bytes(T, B, Hq, c.heads, c.dim, max_pages * c.page), ws, q.device)
    _run(lib().attn_kv8, (q, *cache, cu, lens, table, out, lse, ws),
         (_ptr(q), *qs, c, _ptr(cu), _ptr(lens), _ptr(table), T, B, max_pages, Hq, int(causal), window,
          1.0 / math.sqrt(c.dim) if scale is None else scale, _ptr(out), _ptr(lse), _ptr(ws), wsb), stream)
    return (out, lse) if want_lse or lse is not None else out


@_on_stream
def quantize_weights_group(W: torch.Tensor, group: int = 128, *, Wq=None, s_w=None, stream=None):
    """fp16 weights [N, K] -> packed int4 codes [N, K/2] and fp16 scales [K/group, N], one for
    each output channel and group of inputs."""
    N, K = W.shape
    _need(W, "W", torch.float16)
    if group < 1 or K % group:
        raise ValueError(f"group={group} must divide K={K}")
    if Wq is None:
        Wq = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    if s_w is None:
        s_w = torch.empty((K // group, N), dtype=torch.float16, device=W.device)
    _need(Wq, "Wq", torch.uint8, (N, K // 2))
    _need(s_w, "s_w", torch.float16, (K // group, N))
    _run(lib().sq_quantize_weights_group, (W, Wq, s_w), (_ptr(W), N, K, group, _ptr(Wq), _ptr(s_w)), stream)
    return Wq, s_w


@_on_stream
def w4a16_gemm_frag(X: torch.Tensor, Wf: torch.Tensor, s_w: torch.Tensor, *, Y=None, stream=None):
    """Y = X W^T for fp16 rows X [M, K] and 4-bit weights with group scales: Wf the codes in
    fragment order (weights_to_frag), s_w [K/group, N] fp16 (quantize_weights_group).  Made for
    few rows."""
    M, K = X.shape
    ng, N = s_w.shape
    if ng < 1 or K % ng:
        raise ValueError(f"s_w has {ng} groups, which do not divide K={K}")
    _need(X, "X", torch.float16)
    _need(Wf, "Wf", torch.uint8, _frag_shape(N, K, 4))
    _need(s_w, "s_w", torch.float16, (ng, N))
    if Y is None:
        Y = X.new_empty((M, N))
    else:
        _need(Y, "Y", torch.float16, (M, N))
    _run(lib().w4a16_gemm_frag, (X, Wf, s_w, Y), (_ptr(X), _ptr(Wf), _ptr(s_w), M, N, K, K // ng, _ptr(Y)), stream)
    return Y


ACTIVATIONS = {"none": 0, "relu": 1, "relu2": 2, "silu": 3, "gelu": 4, "gelu_tanh": 5}
_workspace_bytes = functools.lru_cache(maxsize=4096)(gemm_workspace_bytes)      # of sizes alone


def _at(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _epilogue(M: int, N: int, like: torch.Tensor, bias, act: str, glu: bool, residual, Y, dtype):
    """Checks what a fused epilogue takes; returns it and Y."""
    if glu and N % 16:
        raise ValueError(f"glu needs N % 16 == 0, got N={N}")
    shape = (M, N // 2 if glu else N)
    if dtype is None:
        dtype = Y.dtype if Y is not None else residual.dtype if residual is not None else torch.float16
    f32 = dtype is torch.float32
    if not f32 and dtype is not torch.float16:
        raise ValueError(f"the output must be torch.float16 or torch.float32, got {dtype}")
    if bias is not None:
        _need(bias, "bias", torch.float16, (N,))
    if residual is not None:
        _need(residual, "residual", dtype, shape)
    if Y is not None:
        _need(Y, "Y", dtype, shape)
    elif residual is not None:
        Y = torch.empty_like(residual)
    else:
        Y = like.new_empty(shape, dtype=dtype)
    return EPILOGUE.pack(_at(bias), _at(residual), _choice(ACTIVATIONS, act, "act"), bool(glu), f32), Y


@_on_stream
def w4a4_linear(Aq: torch.Tensor, s_a: torch.Tensor, Wf: torch.Tensor, s_w: torch.Tensor, *, bias=None,
                act: str = "none", glu: bool = False, residual=None, Y=None, dtype: Optional[torch.dtype] = None, ws=None,
                stream=None, bits: int = 4):
    """w4a4_gemm_frag with bias [N] fp16, activation ("none", "relu", "relu2", "silu", "gelu" or
    "gelu_tanh") and residual in its epilogue: Y = act(t) + residual with t the dequantised
    product plus bias.  glu=True: the rows of W are N/2 gates and then their ups
    (weights_to_frag(glu=True); s_w and bias in the rows' order), Y = act(t_gate) t_up + residual
    [M, N/2].  Y and residual are both fp16 or both fp32 (dtype; default the residual's, else fp16);
    Y may be the residual.  bits=8 takes int8 codes."""
    M, Kc = Aq.shape
    N = s_w.shape[0]
    K = Kc if bits == 8 else 2 * Kc
    _need(Aq, "Aq", torch.int8 if bits == 8 else torch.uint8)
    _need(Wf, "Wf", torch.uint8, _frag_shape(N, K, bits))
    _need(s_a, "s_a", torch.float32, (M,))
    _need(s_w, "s_w", torch.float32, (N,))
    e, Y = _epilogue(M, N, Aq, bias, act, glu, residual, Y, dtype)
    ws, wsb = _ws(_workspace_bytes(M, N, K, bits), ws, Aq.device)
    _run(lib().w8a8_linear if bits == 8 else lib().w4a4_linear, (Aq, s_a, Wf, s_w, bias, residual, Y, ws),
         (Aq.data_ptr(), s_a.data_ptr(), Wf.data_ptr(), s_w.data_ptr(), M, N, K, e, Y.data_ptr(), _ptr(ws), wsb), stream)
    return Y


def w8a8_linear(Aq, s_a, Wf, s_w, **kw):
    return w4a4_linear(Aq, s_a, Wf, s_w, bits=8, **kw)


@_on_stream
def w4a16_linear(X: torch.Tensor, Wf: torch.Tensor, s_w: torch.Tensor, *, bias=None, act: str = "none",
                 glu: bool = False, residual=None, Y=None, dtype: Optional[torch.dtype] = None, stream=None):
    """w4a16_gemm_frag (fp16 rows X [M, K], 4-bit weights, scales s_w [K/group, N]) with the epilogue
    of w4a4_linear.  Made for few rows."""
    M, K = X.shape
    ng, N = s_w.shape
    if ng < 1 or K % ng:
        raise ValueError(f"s_w has {ng} groups, which do not divide K={K}")
    _need(X, "X", torch.float16)
    _need(Wf, "Wf", torch.uint8, _frag_shape(N, K, 4))
    _need(s_w, "s_w", torch.float16, (ng, N))
    e, Y = _epilogue(M, N, X, bias, act, glu, residual, Y, dtype)
    _run(lib().w4a16_linear, (X, Wf, s_w, bias, residual, Y),
         (X.data_ptr(), Wf.data_ptr(), s_w.data_ptr(), M, N, K, K // ng, e, Y.data_ptr()), stream)
    return Y


def _conditions(K: int, gate, scale, shift):
    """(rows, distances between them) of gate, scale and shift, [seqs, K], or [K] or [1, K] for all; None: not
    given."""
    seqs, strides = 1, []
    for t, name in ((gate, "gate"), (scale, "scale"), (shift, "shift")):
        if t is None:
            strides.append(0)
            continue
        if not t.is_cuda or t.dtype is not torch.float16 or t.dim() not in (1, 2) or t.shape[-1] != K:
            raise ValueError(f"{name} must be a torch.float16 device tensor of shape [K={K}] or [seqs, K]")
        n = t.shape[0] if t.dim() == 2 else 1
        if t.stride(-1) != 1:
            raise ValueError(f"{name} must be dense in its last dimension")
        if n == 0 or (n > 1 and seqs > 1 and n != seqs):
            raise ValueError("gate, scale and shift must have the same number of rows, or one")
        seqs = max(seqs, n)
        strides.append(t.stride(0) if n > 1 else 0)
    return seqs, strides


_NO_ROWS = (0, (0, 0, 0))


def _norm(h, y, weight, post_weight, gate, alpha, scale, shift, seq, eps, center, h_out, X, codes, s, state, d_m, d_u,
          bits, stream):
    """One sq_norm call on checked outputs; returns h_out (h itself without y)."""
    M, K = shape = h.shape
    dt = h.dtype
    f32 = dt is torch.float32
    if not f32 and dt is not torch.float16:
        raise ValueError(f"h must be torch.float16 or torch.float32, got {dt}")
    _need(h, "h", dt)
    if y is not None:
        _need(y, "y", torch.float16, shape)
    elif post_weight is not None or gate is not None:
        raise ValueError("post_weight and gate need y")
    if weight is not None:
        _need(weight, "weight", torch.float16, (K,))
    if post_weight is not None:
        _need(post_weight, "post_weight", torch.float16, (K,))
    if state is not None:
        _need(state, "state", torch.uint8, (M,))
    if seq is not None:
        _need(seq, "seq", torch.int32, (M,))
    seqs, rows = _NO_ROWS if gate is None and scale is None and shift is None else _conditions(K, gate, scale, shift)
    if seqs > 1 and seq is None and M > 0:
        raise ValueError("seq is required where gate, scale and shift have several rows")
    if h_out is not None:
        _need(h_out, "h_out", dt, shape)
    elif y is not None:
        h_out = torch.empty_like(h)
    a = NORM_ARGS.pack(h.data_ptr(), _at(y), _at(post_weight), _at(gate), _at(scale), _at(shift), *rows, _at(seq),
                       _at(weight), _at(state), _at(h_out), _at(X), _at(codes), _at(s), eps, alpha, seqs, f32, bool(center),
                       bits, d_m, d_u)
    _run(lib().sq_norm, (h, y, weight, post_weight, gate, scale, shift, seq, state, h_out, X, codes, s), (a, M, K), stream)
    return h if h_out is None else h_out


@_on_stream
def norm(h: torch.Tensor, y: Optional[torch.Tensor] = None, *, weight=None, post_weight=None, gate=None,
         alpha: float = 1.0, scale=None, shift=None, seq=None, eps: float = 1e-6, center: bool = False, out=None,
         h_out=None, stream=None):
    """The block output y [M, K] onto the residual stream h [M, K] (fp16 or fp32), and the norm of
    the sum: h' = h + alpha gate y (y normed itself with post_weight), X = norm(h') weight (1 + scale)
    + shift, fp16.  RMS norm, or with center=True the mean taken off.  gate, scale and shift are
    [seqs, K] fp16 (rows any multiple of 8 apart) of which token i takes row seq[i], or [K] for all tokens.  Without y
    h' is h.  Returns (X, h'); h_out may be h."""
    if out is None:
        out = torch.empty_like(h, dtype=torch.float16)
    else:
        _need(out, "out", torch.float16, h.shape)
    return out, _norm(h, y, weight, post_weight, gate, alpha, scale, shift, seq, eps, center, h_out, out, None, None, None,
                      0, 0, 0, stream)


@_on_stream
def norm_quant(h: torch.Tensor, y: Optional[torch.Tensor] = None, *, state=None, d_m: Optional[int] = None,
               d_u: Optional[int] = None, weight=None, post_weight=None, gate=None, alpha: float = 1.0, scale=None,
               shift=None, seq=None, eps: float = 1e-6, center: bool = False, Aq=None, s_a=None, h_out=None, out=None,
               stream=None, bits: int = 4):
    """norm straight into the codes of the next product (P folded): the rows, unrounded, gated by
    their state as in sgat_quant_act and quantised as by sgat_quantize.  Returns (Aq, s_a, h'); out
    takes the fp16 rows too."""
    M, K = h.shape
    dt, kw = _codes_spec(bits, K)
    if Aq is None:
        Aq = h.new_empty((M, kw), dtype=dt)
    else:
        _need(Aq, "Aq", dt, (M, kw))
    if s_a is None:
        s_a = h.new_empty((M,), dtype=torch.float32)
    else:
        _need(s_a, "s_a", torch.float32, (M,))
    if out is not None:
        _need(out, "out", torch.float16, (M, K))
    h_out = _norm(h, y, weight, post_weight, gate, alpha, scale, shift, seq, eps, center, h_out, out, Aq, s_a, state,
                  K // 32 if d_m is None else d_m, K // 32 if d_u is None else d_u, bits, stream)
    return Aq, s_a, h_out
