"""Host-side refusals of the products with a fused epilogue and of the norms: every bad
argument is turned down before anything touches a device."""
import os
import subprocess

import pytest
import torch

import paper_2606_04945_amd as sq
from paper_2606_04945_amd import _lib as L

FAKE = 1 << 20          # a 16-byte aligned non-null address; never dereferenced on these paths
BAD = FAKE + 2
FAR = 1 << 40
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return L.lib()


def epilogue(**kw):
    f = dict(bias=0, residual=0, act=0, glu=0, f32=0)
    f.update(kw)
    return L.EPILOGUE.pack(*(f[n] for n in L.EPILOGUE_FIELDS))


def linear(lib, name, e=None, **kw):
    a = dict(A=FAKE, s_a=FAKE + (1 << 16), Wf=FAKE + (2 << 16), s_w=FAKE + (3 << 16), M=4, N=32, K=128, e=e, Y=FAR, ws=None,
             wsb=0)
    a.update(kw)
    return getattr(lib, name)(*a.values(), None)


def w4a16(lib, e=None, **kw):
    a = dict(X=FAKE, Wf=FAKE + (1 << 16), s_w=FAKE + (2 << 16), M=4, N=32, K=128, group=64, e=e, Y=FAR)
    a.update(kw)
    return lib.w4a16_linear(*a.values(), None)


@pytest.mark.parametrize("name", ["w4a4_linear", "w8a8_linear", "w4a16_linear"])
def test_epilogues(lib, name):
    call = w4a16 if name == "w4a16_linear" else lambda lib, e=None, **kw: linear(lib, name, e, **kw)  # noqa: E731
    for kw in (dict(act=-1), dict(act=6), dict(residual=FAR + 16), dict(residual=FAR - 16), dict(bias=FAR)):
        assert call(lib, epilogue(**kw)) == L.SQ_ERR_SHAPE, kw
    assert call(lib, epilogue(glu=1), N=24) == L.SQ_ERR_SHAPE
    assert call(lib, N=(1 << 22) + 8, K=64 if call is not w4a16 else 128) == L.SQ_ERR_SHAPE
    assert b"2^22" in lib.sq_last_error()
    assert call(lib, epilogue(glu=1), N=24, M=0) == L.SQ_ERR_SHAPE
    for kw in (dict(bias=BAD), dict(residual=BAD)):
        assert call(lib, epilogue(**kw)) == L.SQ_ERR_ALIGN, kw
    for kw in (dict(N=12), dict(K=100), dict(K=0), dict(M=-1), dict(N=-8), dict(M=1 << 23)):
        assert call(lib, **kw) == L.SQ_ERR_SHAPE, kw
    for kw in (dict(Wf=None), dict(s_w=None), dict(Y=None)):
        assert call(lib, **kw) == L.SQ_ERR_NULL, kw
    for kw in (dict(Wf=BAD), dict(s_w=BAD), dict(Y=FAR + 2)):
        assert call(lib, **kw) == L.SQ_ERR_ALIGN, kw
    # Y on an input, or ending in one
    for kw in (dict(Y=FAKE), dict(Y=FAKE - 16), dict(Wf=FAR + 64), dict(s_w=FAR)):
        assert call(lib, **kw) == L.SQ_ERR_SHAPE, kw
    assert call(lib, M=0) == L.SQ_OK and call(lib, N=0) == L.SQ_OK


def test_own_rules(lib):
    assert linear(lib, "w8a8_linear", K=65536 + 64) == L.SQ_ERR_SHAPE
    assert linear(lib, "w4a4_linear", M=96, N=4096, K=12288) == L.SQ_ERR_WORKSPACE
    assert linear(lib, "w4a4_linear", M=96, N=4096, K=12288, ws=BAD, wsb=1 << 40) == L.SQ_ERR_ALIGN
    assert linear(lib, "w4a4_linear", s_a=None) == L.SQ_ERR_NULL
    assert linear(lib, "w4a4_linear", M=1 << 20, N=8, K=131072) == L.SQ_ERR_SHAPE      # operands under 2 GiB
    for g in (0, 16, 48, 96, 256, -64):
        assert w4a16(lib, group=g) == L.SQ_ERR_SHAPE, g


def test_weights_of_pairs(lib):
    f, f8 = lib.sq_weights_to_frag_glu, lib.sq_weights_to_frag_glu_w8
    for g, K in ((f, 128), (f8, 128)):
        assert g(FAKE, 24, K, FAR, None) == L.SQ_ERR_SHAPE and g(FAKE, -16, K, FAR, None) == L.SQ_ERR_SHAPE
        assert g(FAKE, 32, 100, FAR, None) == L.SQ_ERR_SHAPE and g(FAKE, 32, K, FAKE + 64, None) == L.SQ_ERR_SHAPE
        assert g(None, 32, K, FAR, None) == L.SQ_ERR_NULL and g(FAKE, 32, K, FAR + 8, None) == L.SQ_ERR_ALIGN
        assert g(None, 0, K, None, None) == L.SQ_OK
    assert f8(FAKE, 32, 65536 + 64, FAR, None) == L.SQ_ERR_SHAPE
    assert f(FAKE, 1 << 20, 8192, FAR, None) == L.SQ_ERR_SHAPE


def norm(lib, M=4, K=64, **kw):
    f = dict.fromkeys(L.NORM_FIELDS, 0)
    f.update(h=FAKE, X=FAR, eps=1e-6, alpha=1.0)
    f.update(kw)
    return lib.sq_norm(L.NORM_ARGS.pack(*(f[n] or 0 for n in L.NORM_FIELDS)), M, K, None)


def test_norm(lib):
    codes = dict(X=None, codes=FAR, s=FAR + (1 << 20), bits=4, d_m=2, d_u=2)
    rows = dict(seqs=3, scale=2 * FAKE, shift=3 * FAKE, scale_row=64, shift_row=128)
    assert lib.sq_norm(None, 4, 64, None) == L.SQ_ERR_NULL
    for kw in (dict(K=0), dict(K=12), dict(K=32776), dict(K=-8), dict(M=-1), dict(M=4194241), dict(eps=0.0), dict(eps=1e-31),
               dict(eps=-1.0),
               dict(eps=NAN), dict(eps=INF), dict(alpha=NAN), dict(alpha=INF),
               {**rows, "seqs": 0}, {**rows, "seqs": -1}, {**rows, "scale_row": 56}, {**rows, "shift_row": 68},
               {**rows, "shift_row": -64}, {**rows, "scale_row": 1 << 40},
               {**codes, "bits": 0}, {**codes, "bits": 6}, {**codes, "K": 72}, {**codes, "d_m": -1}, {**codes, "d_u": 62},
               # outputs on inputs and on each other
               dict(X=FAKE), dict(h_out=FAKE + 16), dict(h_out=FAKE, y=FAKE), dict(h_out=FAKE, y=FAKE, f32=1),
               dict(h_out=FAKE, weight=FAKE), dict(h_out=FAR + 32), dict(y=FAR), dict(weight=FAR + 16),
               {**rows, "scale": FAR - 368}, {**codes, "state": FAR}, {**codes, "s": FAR}, {**codes, "h_out": FAR}):
        assert norm(lib, **kw) == L.SQ_ERR_SHAPE, kw
    for kw in (dict(h=None), dict(X=None), {**codes, "s": None}, {**codes, "codes": None}, dict(X=FAR, s=FAKE << 2, bits=4),
               dict(gate=2 * FAKE, seqs=1), dict(y_weight=2 * FAKE)):
        assert norm(lib, **kw) == L.SQ_ERR_NULL, kw
    for kw in (dict(h=BAD), dict(X=FAR + 8), dict(y=BAD), dict(weight=BAD), dict(h_out=BAD), {**rows, "seq": BAD},
               {**rows, "scale": BAD}, {**codes, "codes": FAR + 4}, {**codes, "s": FAR + (1 << 20) + 4}):
        assert norm(lib, **kw) == L.SQ_ERR_ALIGN, kw
    assert norm(lib, M=0, h=None) == L.SQ_OK
    assert norm(lib, M=0, **{**rows, "scale_row": 0, "shift_row": 0}) == L.SQ_OK     # one row for all


def test_binding_refuses():
    h = torch.zeros(2, 64, dtype=torch.float16)
    for call in (lambda: sq.norm(h), lambda: sq.norm_quant(h), lambda: sq.w4a16_linear(h, None, torch.zeros(1, 16)),
                 lambda: sq.w4a4_linear(torch.zeros(2, 32, dtype=torch.uint8), None, None, torch.zeros(16))):
        with pytest.raises((ValueError, RuntimeError)):
            call()


def test_struct_layouts(tmp_path):
    """The binding packs the header's structures: every field where the C compiler has it."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for struct, fields in (("sq_epilogue", L.EPILOGUE_FIELDS), ("sq_norm_args", L.NORM_FIELDS)):
        lines.append(f'printf("%zu\\n", sizeof({struct}));')
        lines += [f'printf("%zu %zu\\n", offsetof({struct}, {f}), sizeof((({struct}*)0)->{f}));' for f in fields]
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include "starquant.h"\nint main(void) {' + "\n".join(lines)
                                  + "return 0; }")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    told = iter(subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.splitlines())
    for packer, fields in ((L.EPILOGUE, L.EPILOGUE_FIELDS), (L.NORM_ARGS, L.NORM_FIELDS)):
        assert packer.size == int(next(told))
        for i, f in enumerate(fields):
            at, size = map(int, next(told).split())
            one = packer.pack(*(1.0 if j == i and f in ("eps", "alpha") else int(j == i) for j in range(len(fields))))
            assert any(one[at:at + size]) and not any(one[:at]) and not any(one[at + size:]), f
