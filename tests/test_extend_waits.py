"""The extend kernels' row loads into LDS are assembly statements too (see test_prefill_waits.py): the compiler inserts
no wait state between a write of m0 and the load that reads it, and none behind a vector instruction that wrote an SGPR
of the load's address. This compiles the kernels to assembly and counts both."""
import os
import subprocess

from paper_2609_08368_amd import build
from tests.test_prefill_waits import load_faults


def test_waits_of_the_row_loads(tmp_path):
    out = os.path.join(tmp_path, "extend.s")
    subprocess.run([*build.compiler(), "--offload-device-only", "-S", os.path.join(build.CSRC, "extend.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        loads, found = load_faults(f.read())
    assert loads > 0 and not found, f"{len(found)} of {loads}\n" + "\n".join(found[:20])
