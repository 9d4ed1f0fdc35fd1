"""The build's options leave the compiler's warnings about assembly statements on (one statement turns its own off)."""
import os
import subprocess

from paper_2609_08368_amd import build

SOURCE = """
#include <hip/hip_runtime.h>
__global__ void f(int* x) { int y; asm volatile("s_mov_b32 exec_hi, 0" ::: "exec"); y = threadIdx.x; x[y] = y; }
"""


def test_a_statement_that_sets_a_reserved_register_is_warned_of(tmp_path):
    path = os.path.join(tmp_path, "f.hip")
    with open(path, "w") as f:
        f.write(SOURCE)
    res = subprocess.run([*build.compiler(), "--offload-device-only", "-S", path, "-o", path + ".s"], capture_output=True,
                         text=True)
    assert res.returncode == 0 and "-Winline-asm" in res.stderr, res.stderr
