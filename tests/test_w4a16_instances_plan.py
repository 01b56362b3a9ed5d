"""The weight-only plan, asked which instance each shape of test_gpu_w4a16_instances.py takes, and
whether any shape takes one that is not among them."""
import ctypes
import os
import subprocess

from test_gpu_w4a16_instances import INSTANCES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "w4a16_plan.hpp"
extern "C" void plan(int M, int N, int* o) {
    const sq::W4a16Plan p = sq::w4a16_plan(M, N);
    o[0] = p.tm; o[1] = p.ng; o[2] = p.waves; o[3] = p.lines;
}
"""


def test_every_instance_is_tested(tmp_path):
    (tmp_path / "shim.cpp").write_text(SHIM)
    so = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2606_04945_amd", "csrc"), str(tmp_path / "shim.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)

    def plan(M, N):
        o = (ctypes.c_int * 4)()
        lib.plan(M, N, o)
        return (o[0], o[1], o[2], bool(o[3]))

    for name, (M, N) in INSTANCES.items():
        assert plan(M, N) == name, (M, N, plan(M, N))
    taken = {plan(M, N) for M in (*range(1, 66), 100, 130, 1000, 65535 * 16) for N in (*range(8, 66000, 56), 126464, 1 << 20)}
    assert taken == set(INSTANCES), taken ^ set(INSTANCES)
