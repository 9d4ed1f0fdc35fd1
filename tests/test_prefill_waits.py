"""The prefill kernel's score products and its loads into LDS are assembly statements, which the compiler does not
know as matrix and memory instructions, so it inserts none of the wait states that they need around them. This
compiles the kernel to assembly and counts them. For the 8-pass v_mfma_f32_32x32x16_bf16:

* a result read or overwritten by anything but the next product of its chain: 11 wait states,
* an addend overwritten: 7,
* an operand written by a vector instruction before: 2.

For a load, 5 after a vector instruction that wrote an SGPR of its address, and 1 after a write of m0.

An instruction counts as one (a matrix instruction as one too, though it takes longer), ``s_nop n`` as n + 1.
"""
import os
import re
import subprocess

import pytest

from paper_2609_08368_amd import build

READ, ADDEND, OPERAND, SGPR, M0 = 11, 7, 2, 5, 1
NAME = "v_mfma_f32_32x32x16_bf16"


def registers(text):
    out = []
    for m in re.finditer(r"\b([vas])\[(\d+):(\d+)\]|\b([vas])(\d+)\b", text):
        out.append((m[1], int(m[2]), int(m[3])) if m[1] else (m[4], int(m[5]), int(m[5])))
    return out


def meet(a, b):
    return a[0] == b[0] and a[1] <= b[2] and b[1] <= a[2]


def any_meet(xs, ys):
    return any(meet(x, y) for x in xs for y in ys)


def instructions(text):
    """(mnemonic, operands) of every instruction, in the order of the file."""
    out = []
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        if line and not line.startswith((".", "//")) and not line.endswith(":"):
            name, _, rest = line.partition(" ")
            out.append((name, [o.strip() for o in rest.split(",")] if rest.strip() else []))
    return out


def states(ins):
    return int(ins[1][0]) + 1 if ins[0] == "s_nop" else 1


def faults(text):
    """Number of score products, and a line for each of their waits that is too short."""
    code = instructions(text)
    found, products = [], 0
    for i, (name, ops) in enumerate(code):
        if name != NAME or not ops[0].startswith("v"):
            continue                       # (accumulators of the compiler's own products are in a registers)
        products += 1
        dst, addend = registers(ops[0]), registers(ops[3]) if ops[3].startswith("v") else []
        waited = 0
        for y, y_ops in code[i + 1:]:
            if waited >= READ:
                break
            if y.startswith("s_"):
                waited += states((y, y_ops))
                continue
            used = registers(", ".join(y_ops))
            if y.startswith("v_mfma") and any_meet(used, dst):
                chained = y == NAME and not any_meet(registers(", ".join(y_ops[1:3])), dst)
                if not chained:
                    found.append(f"{waited} states: {name} {ops} -> {y} {y_ops}")
                break
            if any_meet(used, dst):
                found.append(f"{waited} states: {name} {ops} -> {y} {y_ops}")
                break
            if waited < ADDEND and y.startswith("v_") and not y.startswith("v_mfma") \
                    and any_meet(registers(y_ops[0]), addend):
                found.append(f"{waited} states: addend of {name} {ops} -> {y} {y_ops}")
            waited += 1
        waited = 0
        for y, y_ops in reversed(code[max(0, i - 4):i]):
            if waited >= OPERAND:
                break
            if y.startswith("v_") and not y.startswith("v_mfma") \
                    and any_meet(registers(y_ops[0]), registers(", ".join(ops[1:]))):
                found.append(f"{waited} states: {y} {y_ops} -> {name} {ops}")
            waited += states((y, y_ops))
    return products, found


def load_faults(text):
    """Number of loads into LDS, and a line for each of their waits that is too short."""
    code = instructions(text)
    found, loads = [], 0
    for i, (name, ops) in enumerate(code):
        if not name.startswith("global_load_lds"):
            continue
        loads += 1
        address = [r for r in registers(", ".join(ops)) if r[0] == "s"]
        waited = 0
        for y, y_ops in reversed(code[max(0, i - SGPR):i]):
            if waited >= SGPR:
                break
            writes = registers(y_ops[0]) if y_ops and y.startswith("v_") else []
            if any_meet(writes, address) or (waited < M0 and y_ops and y_ops[0] == "m0"):
                found.append(f"{waited} states: {y} {y_ops} -> {name} {ops}")
            waited += states((y, y_ops))
    return loads, found


CHAIN = """
	v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], a[0:3], 0
	v_add_f32_e32 v60, v61, v62
	v_mfma_f32_32x32x16_bf16 v[0:15], v[44:47], a[4:7], v[0:15]
	v_mfma_f32_32x32x16_bf16 v[16:31], v[48:51], a[8:11], v[0:15]
"""


@pytest.mark.parametrize("tail, number", [
    ("s_nop 10\n v_mov_b32_e32 v70, v16", 0),
    ("s_nop 9\n v_mov_b32_e32 v70, v16", 1),
    ("s_nop 9\n v_add_f32_e32 v70, v1, v16", 1),
    ("s_nop 6\n v_mov_b32_e32 v3, v70", 0),
    ("s_nop 5\n v_mov_b32_e32 v3, v70", 1),
    ("v_mov_b32_e32 v90, v91\n s_nop 8", 0),
    ("s_nop 10\n v_accvgpr_write_b32 a0, v70\n s_nop 0\n v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], a[0:3], 0", 1),
    ("s_nop 10\n v_accvgpr_write_b32 a0, v70\n s_nop 1\n v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], a[0:3], 0", 0),
])
def test_the_count(tail, number):
    assert len(faults(CHAIN + tail)[1]) == number


@pytest.mark.parametrize("code, number", [
    ("v_readlane_b32 s5, v253, 49\n s_nop 3", 1), ("v_readlane_b32 s5, v253, 49\n s_nop 4", 0),
    ("s_add_u32 s5, s5, s6", 0), ("v_readfirstlane_b32 s4, v1\n v_mov_b32_e32 v9, v8\n s_nop 2", 1),
    ("s_mov_b32 m0, s7", 1), ("s_mov_b32 m0, s7\n s_nop 0", 0)])
def test_the_count_of_loads(code, number):
    loads, found = load_faults(code + "\n global_load_lds_dwordx4 v2, s[4:5]")
    assert loads == 1 and len(found) == number


def test_waits_of_the_kernel(tmp_path):
    out = os.path.join(tmp_path, "prefill.s")
    subprocess.run([*build.compiler(), "--offload-device-only", "-S", os.path.join(build.CSRC, "prefill.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    for count, found in (faults(text), load_faults(text)):
        assert count > 0 and not found, "\n".join(found)
