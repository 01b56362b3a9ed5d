"""Which kernel a weight-only product takes, asked of the planning code compiled with g++."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_w4a16 import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04945_amd", "csrc")
SHIM = r"""
#include "w4a16_plan.hpp"
extern "C" void plan(int M, int N, int* o) {
    const sq::W4a16Plan p = sq::w4a16_plan(M, N);
    o[0] = p.tm; o[1] = p.ng; o[2] = p.waves;
}
"""
KERNELS = {(1, 1), (1, 2), (1, 3), (1, 4), (1, 5), (2, 1), (2, 2), (4, 1), (4, 2)}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("w4a16_plan")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", so],
                   check=True)
    lib = ctypes.CDLL(so)

    def ask(M, N):
        o = (ctypes.c_int * 3)()
        lib.plan(M, N, o)
        return tuple(o)
    return ask


def test_only_kernels_that_exist(plan):
    for M in (*range(1, 70), 100, 1000, 65535 * 16):
        for N in (*range(8, 3000, 56), 4096, 12288, 24576, 37888, 126464, 1 << 20):
            tm, ng, waves = plan(M, N)
            assert (tm, ng) in KERNELS and waves in (4, 8) and 16 * tm >= min(M, 64) - (M > 64) * 16


def test_every_kernel_is_tested(plan):
    assert {plan(M, N)[:2] for M, N, _, _ in SHAPES} == KERNELS
    assert {plan(M, N)[2] for M, N, _, _ in SHAPES} == {4, 8}


def test_measured_shapes_take_the_faster_side(plan):
    assert plan(16, 37888) == (1, 5, 4)
    assert plan(1, 24576)[1] in (2, 3) and plan(1, 4096) == (1, 1, 8) and plan(5, 3584) == (1, 1, 8)
