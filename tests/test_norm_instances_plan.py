"""The norms' launch plan asked which share of a row each shape of test_gpu_norm_instances.py takes: every
one that the library holds, each with and without options, as rows and as codes."""
import ctypes
import os
import subprocess

from test_gpu_norm_instances import INSTANCES
from test_norm_plan import CSRC, SHIM, instances


def test_every_instance_is_run(tmp_path):
    (tmp_path / "s.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "s.cpp"), "-o",
                    str(tmp_path / "s.so")], check=True)
    plan = ctypes.CDLL(str(tmp_path / "s.so")).plan
    for (waves, nv), shapes in INSTANCES.items():
        for M, K in shapes:
            assert plan(M, K) == 8 * waves + nv and K % 64 == 0, (M, K)      # (codes need K % 64 == 0)
    assert {8 * waves + nv for waves, nv in INSTANCES} == instances()
    # what the kernel is an instance of beside these: type of the stream, options, width of the codes
    src = open(os.path.join(CSRC, "norm.hip")).read()
    assert "template <int NV, bool F32, int WAVES, bool FULL, int BITS>" in src
