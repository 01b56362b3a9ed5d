"""The norms' launch plan (host C++ without HIP): every row fits its waves, and every instance that the
library holds is reached."""
import ctypes
import os
import re
import subprocess

from test_gpu_norm import KS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_04945_amd", "csrc")
SHIM = """#include "norm_plan.hpp"
extern "C" int plan(int M, int K) { const sq::NormPlan p = sq::norm_plan(M, K); return p.waves * 8 + p.nv; }"""
ROWS = (1, 5, 512, 513, 1024, 1025, 20000)


def instances():
    src = open(os.path.join(CSRC, "norm.hip")).read()
    return {int(w) + int(v) for w, v in re.findall(r"case (\d+) \+ (\d+): return launch", src)}


def test_plan(tmp_path):
    (tmp_path / "s.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "s.cpp"), "-o",
                    str(tmp_path / "s.so")], check=True)
    plan = ctypes.CDLL(str(tmp_path / "s.so")).plan
    seen = set()
    for K in range(8, 32769, 8):
        for M in ROWS:
            p = plan(M, K)
            seen.add(p)
            assert 64 * (p // 8) * (p % 8) * 8 >= K and p // 8 <= 16, (M, K)
    assert seen == instances()
    # the widths of the GPU tests reach every instance, those of many rows with the row counts below
    assert {plan(M, K) for K in KS for M in (5, 1100)} == seen
