"""The wait states of test_prefill_waits.py over every path of the compiled prefill kernel, branches and the step loops'
back edges included, and as long as the compiler itself waits: for the same product written as a builtin it leaves 12
states before its result is read (one more than that file asks for), 7 before its addend is overwritten, and 2 between
an operand's last writer and the product."""
import os
import subprocess

import pytest

from paper_2609_08368_amd import build
from tests.test_prefill_waits import CHAIN, M0, NAME, SGPR, any_meet, registers, states

READ, ADDEND, OPERAND = 12, 7, 2


class Code:
    """Instructions (mnemonic, operands) of a file of assembly with those that may follow and precede each."""

    def __init__(self, text):
        self.ins, labels = [], {}
        for line in text.splitlines():
            line = line.split(";")[0].strip()
            if line.endswith(":"):
                labels[line[:-1]] = len(self.ins)
            elif line and not line.startswith((".", "//")):
                name, _, rest = line.partition(" ")
                name, _, tab = name.partition("\t")
                rest = (tab + " " + rest).strip()
                self.ins.append((name, [o.strip() for o in rest.split(",")] if rest else []))
        self.next = [[] for _ in self.ins]
        self.before = [[] for _ in self.ins]
        for i, (name, ops) in enumerate(self.ins):
            to = [i + 1] if name not in ("s_branch", "s_endpgm", "s_setpc_b64") else []
            if name == "s_branch" or name.startswith("s_cbranch"):
                to.append(labels[ops[0]])
            self.next[i] = [t for t in to if t < len(self.ins)]
            for t in self.next[i]:
                self.before[t].append(i)

    def walk(self, start, step, limit, visit):
        """Calls visit(instruction, states waited) along every path from `start` until it returns True or `limit` states
        have passed."""
        seen, todo = {}, [(t, 0) for t in step[start]]
        while todo:
            i, waited = todo.pop()
            if waited >= limit or seen.get(i, limit) <= waited:
                continue
            seen[i] = waited
            if not visit(self.ins[i], waited):
                todo += [(t, waited + states(self.ins[i])) for t in step[i]]


def product_faults(text):
    code, found, products = Code(text), [], 0
    for i, (name, ops) in enumerate(code.ins):
        if name != NAME or not ops[0].startswith("v"):
            continue
        products += 1
        dst, addend = registers(ops[0]), registers(ops[3]) if ops[3].startswith("v") else []

        def after(y, waited):
            if y[0].startswith("s_"):
                return False
            used = registers(", ".join(y[1]))
            if any_meet(used, dst):
                if not (y[0] == NAME and not any_meet(registers(", ".join(y[1][1:3])), dst)):
                    found.append(f"{waited} states: {name} {ops} -> {y}")
                return True
            if waited < ADDEND and y[0].startswith("v_") and not y[0].startswith("v_mfma") \
                    and any_meet(registers(y[1][0]), addend):
                found.append(f"{waited} states: addend of {name} {ops} -> {y}")
            return False

        def behind(y, waited):
            if y[0].startswith("v_") and not y[0].startswith("v_mfma") \
                    and any_meet(registers(y[1][0]), registers(", ".join(ops[1:]))):
                found.append(f"{waited} states: {y} -> {name} {ops}")
            return False

        code.walk(i, code.next, READ, after)
        code.walk(i, code.before, OPERAND, behind)
    return products, found


def load_faults(text):
    code, found, loads = Code(text), [], 0
    for i, (name, ops) in enumerate(code.ins):
        if not name.startswith("global_load_lds"):
            continue
        loads += 1
        address = [r for r in registers(", ".join(ops)) if r[0] == "s"]

        def behind(y, waited):
            writes = registers(y[1][0]) if y[1] and y[0].startswith("v_") else []
            if any_meet(writes, address) or (waited < M0 and y[1] and y[1][0] == "m0"):
                found.append(f"{waited} states: {y} -> {name} {ops}")
            return False

        code.walk(i, code.before, SGPR, behind)
    return loads, found


def assembly(source, out):
    subprocess.run([*build.compiler(), "--offload-device-only", "-S", source, "-o", out], check=True, capture_output=True)
    with open(out) as f:
        return f.read()


LOOP = """
loop:
	{head}
	v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], a[0:3], 0
	{tail}
	s_cbranch_scc1 loop
	s_endpgm
"""


@pytest.mark.parametrize("head, tail, number", [
    ("v_mov_b32_e32 v70, v3", "s_nop 10", 0), ("v_mov_b32_e32 v70, v3", "s_nop 9", 1),
    ("s_nop 0", "v_accvgpr_write_b32 a1, v80", 0), ("", "v_accvgpr_write_b32 a1, v80", 1)])
def test_the_count_over_a_back_edge(head, tail, number):
    assert len(product_faults(LOOP.format(head=head, tail=tail))[1]) == number


@pytest.mark.parametrize("tail, number", [
    ("s_nop 11\n v_mov_b32_e32 v70, v16", 0), ("s_nop 10\n v_mov_b32_e32 v70, v16", 1),
    ("s_nop 6\n v_mov_b32_e32 v3, v70", 0), ("s_nop 5\n v_mov_b32_e32 v3, v70", 1),
    ("s_cbranch_vccz over\n s_nop 15\nover:\n s_nop 9\n v_mov_b32_e32 v70, v16", 1),
    ("s_cbranch_vccz over\n s_nop 15\nover:\n s_nop 10\n v_mov_b32_e32 v70, v16", 0)])
def test_the_count(tail, number):
    assert len(product_faults(CHAIN + tail)[1]) == number


@pytest.mark.parametrize("code, number", [
    ("s_mov_b32 m0, s7\n s_cbranch_scc0 to\n s_nop 0\nto:", 0), ("s_branch to\n s_mov_b32 m0, s7\nto:", 1),
    ("v_readlane_b32 s5, v3, 4\n s_cbranch_scc0 to\n s_nop 3\nto:", 1),
    ("v_readlane_b32 s5, v3, 4\n s_cbranch_scc0 to\nto:\n s_nop 3", 0)])
def test_the_count_of_loads(code, number):
    loads, found = load_faults(code + "\n global_load_lds_dwordx4 v2, s[4:5]")
    assert loads == 1 and len(found) == number


BUILTINS = """
#include <hip/hip_runtime.h>
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
__global__ void result(const bf16x8* a, const bf16x8* b, float* o) {
  f32x16 c = {};
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[threadIdx.x], b[threadIdx.x], c, 0, 0, 0);
  o[threadIdx.x] = c[0] + 1.f;
}
__global__ void operand(const bf16x8* a, const uint4* b, float* o, unsigned z) {
  uint4 q = b[threadIdx.x];
  f32x16 c = {};
  q.w += z;
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[threadIdx.x], __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
  o[threadIdx.x] = c[0];
}
"""


def test_the_compiler_waits_as_long(tmp_path):
    source = os.path.join(tmp_path, "builtins.hip")
    with open(source, "w") as f:
        f.write(BUILTINS)
    code = Code(assembly(source, os.path.join(tmp_path, "builtins.s")))
    at = [i for i, (name, _) in enumerate(code.ins) if name == NAME]
    assert len(at) == 2

    def states_until(i, step, hit):
        waited = 0
        while not hit(code.ins[i]):
            waited += states(code.ins[i])
            i += step
        return waited

    for i in at:
        dst, b = registers(code.ins[i][1][0]), registers(", ".join(code.ins[i][1][1:3]))
        reads = lambda y: not y[0].startswith("s_") and any_meet(registers(", ".join(y[1])), dst)
        assert states_until(i + 1, 1, reads) == READ
    writes = lambda y: y[0].startswith("v_") and any_meet(registers(y[1][0]), b)
    assert states_until(at[1] - 1, -1, writes) == OPERAND


def test_waits_of_the_kernel(tmp_path):
    text = assembly(os.path.join(build.CSRC, "prefill.hip"), os.path.join(tmp_path, "prefill.s"))
    for count, found in (product_faults(text), load_faults(text)):
        assert count > 0 and not found, "\n".join(found[:20])
