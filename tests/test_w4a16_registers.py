"""Registers of the weight-only kernels, as the compiler reports them: instances whose CU has to hold two
workgroups leave room for them, whatever the loop around them looks like."""
import os
import re
import subprocess

import pytest

from paper_2606_04945_amd import build as B
from test_gpu_w4a16_instances import INSTANCES

NAME = re.compile(r"w4a16_kernelILi(\d)ELi(\d)ELi(\d+)ELb(\d)E\w*?(Dequant|FusedILb[01]E)")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    obj = str(tmp_path_factory.mktemp("w4a16") / "o.o")
    r = subprocess.run(["hipcc", *B.FLAGS, "-Rpass-analysis=kernel-resource-usage", "-c", "-o", obj,
                        os.path.join(B.CSRC, "w4a16.hip")], capture_output=True, text=True, check=True)
    out = {}
    for block in r.stderr.split("Function Name: ")[1:]:
        m = NAME.search(block.split()[0])
        if m:
            tm, ng, group, lines = (int(x) for x in m.groups()[:4])
            use = {k: int(re.search(k + r": (\d+)", block)[1]) for k in (" VGPRs", "AGPRs", r"Occupancy \[waves/SIMD\]")}
            out[tm, ng, group, bool(lines), m[5]] = use
    return out


def test_every_instance_is_seen(kernels):
    shares = {(tm, ng, lines) for tm, ng, _, lines in INSTANCES}
    assert {k[:2] + k[3:4] for k in kernels} == shares and len(kernels) == 9 * len(shares)


def test_two_workgroups_of_three_groups_of_outputs(kernels):
    """Two of eight waves: four waves a SIMD, 128 registers."""
    for k, use in kernels.items():
        if k[:2] == (1, 3):
            assert use[" VGPRs"] + use["AGPRs"] <= 128 and use[r"Occupancy \[waves/SIMD\]"] >= 4, (k, use)


def test_two_workgroups_of_many_rows_in_groups_of_32(kernels):
    """Two of four waves: two waves a SIMD, 256 registers."""
    for k, use in kernels.items():
        if k[0] == 4 and k[2] == 32:
            assert use[" VGPRs"] + use["AGPRs"] <= 256 and use[r"Occupancy \[waves/SIMD\]"] >= 2, (k, use)
