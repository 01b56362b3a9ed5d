"""The shapes of test_gpu_w4a16_linear_instances.py take the instances that they are named for, at their K and group of
scales; and how the rows of X are read at sizes that were measured either way."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_w4a16_instances import INSTANCES
from test_gpu_w4a16_linear_instances import GROUPS, shape
from test_w4a16_instances_plan import ROOT

SHIM = r"""
#include "w4a16_plan.hpp"
extern "C" void plan(int M, int N, int K, int group, int* o) {
    const sq::W4a16Plan p = sq::w4a16_plan(M, N, K, group);
    o[0] = p.tm; o[1] = p.ng; o[2] = p.waves; o[3] = p.lines;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("w4a16_lines")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2606_04945_amd", "csrc"), str(d / "shim.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)

    def ask(M, N, K, group):
        o = (ctypes.c_int * 4)()
        lib.plan(M, N, K, group, o)
        return o[0], o[1], o[2], bool(o[3])
    return ask


def test_every_instance_is_run(plan):
    for name in INSTANCES:                            # (all that any shape takes)
        for group in GROUPS:
            M, N, K = shape(name, group)
            assert plan(M, N, K, group) == name and N % 16 == 0 and K % group == 0 and K % 64 == 0, (M, N, K, group)


def test_few_steps_read_rows_as_operands(plan):
    for M, N, K, group in ((5, 4096, 4096, 128), (6, 4096, 4096, 128), (5, 4096, 1024, 128), (12, 8192, 1024, 128),
                           (8, 8192, 2048, 128), (5, 2048, 2048, 64), (5, 1024, 8192, 128), (8, 8192, 4096, 32),
                           (5, 12288, 4096, 32), (8, 12288, 4096, 32), (5, 24576, 4096, 32), (4, 3584, 18944, 64)):
        assert not plan(M, N, K, group)[3], (M, N, K, group)


def test_many_steps_read_them_in_whole_lines(plan):
    for M, N, K, group in ((8, 4096, 4096, 128), (8, 4096, 12288, 128), (5, 3584, 18944, 64), (16, 2048, 2048, 128),
                           (8, 1024, 8192, 128), (5, 12288, 4096, 128), (5, 24576, 4096, 64), (5, 16384, 4096, 128),
                           (16, 12288, 4096, 32), (17, 4096, 1024, 32), (64, 4096, 4096, 64)):
        assert plan(M, N, K, group)[3], (M, N, K, group)
