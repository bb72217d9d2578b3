"""Wait states in the built kernels.

A vector memory instruction that reads a scalar register written by a vector
instruction needs five wait states in between, and a load into LDS one after
the write of m0: the hardware does not check, and the compiler does not look
into inline asm.  This reads the instructions of every kernel of the built
library."""
import os
import re
import subprocess

import pytest

import paper_1904_12380_amd as sm

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
SCALAR = re.compile(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc|m0)\b")
CARRY_OUT = ("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_subbrev_co",
             "v_div_scale", "v_mad_u64_u32", "v_mad_i64_i32")
MEMORY = ("buffer_", "global_", "flat_", "scratch_")


def scalars(operand):
    out = set()
    for a, b, one, named in SCALAR.findall(operand):
        if named:
            out.add(named)
        elif one:
            out.add(int(one))
        else:
            out.update(range(int(a), int(b) + 1))
    return out


def written_by_vector(op, operands):
    """Scalar registers that a vector instruction writes."""
    if op.startswith(("v_readfirstlane", "v_readlane")):
        return scalars(operands[0])
    if op.startswith("v_cmp") and not op.startswith("v_cmpx"):
        return scalars(operands[0])
    if op.startswith(CARRY_OUT):
        return scalars(operands[1])
    return set()


def hazards(lines):
    """(kernel, instruction, wait states had, wanted) of every place with too
    few, along the code as it lies."""
    out, kernel, at, vector, m0 = [], None, 0, {}, None
    for line in lines:
        head = re.match(r"^<(.+)>:$", line.strip()) or re.match(r"^[0-9a-f]+ <(.+)>:$", line)
        if head:
            if not head.group(1).startswith("L"):
                kernel, vector, m0 = head.group(1), {}, None
            continue
        text = line.split("//")[0].strip()
        if not text or kernel is None:
            continue
        op, _, rest = text.partition(" ")
        operands = [x.strip() for x in re.split(r",(?![^\[]*\])", rest)]
        if op.startswith(MEMORY):
            for reg in set().union(*map(scalars, operands)):
                if reg in vector and at - vector[reg] - 1 < 5:
                    out.append((kernel, text, at - vector[reg] - 1, 5))
            if " lds" in text and m0 is not None and at - m0 - 1 < 1:
                out.append((kernel, text, at - m0 - 1, 1))
        if op.startswith("v_"):
            for reg in written_by_vector(op, operands):
                vector[reg] = at
        elif op.startswith("s_") and operands[0]:
            if not op.startswith(("s_cmp", "s_bitcmp", "s_waitcnt", "s_nop", "s_branch", "s_cbranch")):
                for reg in scalars(operands[0]):  # a scalar write: no such hazard
                    vector.pop(reg, None)
                if operands[0] == "m0":
                    m0 = at
        if op in ("s_branch", "s_endpgm", "s_setpc_b64"):
            vector, m0 = {}, None  # nothing runs on into what follows
        at += int(rest) + 1 if op == "s_nop" else 1
    return out


def instructions(tmp_path):
    """The listing of each code object of the built library."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    link = tmp_path / "lib.so"
    link.symlink_to(sm.LIB_PATH)
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    objects = sorted(p for p in os.listdir(tmp_path) if "gfx950" in p)
    assert len(objects) >= 8
    for name in objects:
        done = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp_path,
                              check=True, capture_output=True, text=True)
        yield name, done.stdout.splitlines()


def test_the_reader_sees_a_missing_wait():
    code = ["<k_one>:", "v_readfirstlane_b32 s20, v3", "s_mov_b32 s23, 0x27000", "s_mov_b32 m0, s4",
            "{}", "buffer_load_dwordx4 v2, s[20:23], 0 offen lds"]
    for nop, bad in (("s_nop 0", 1), ("s_nop 1", 1), ("s_nop 2", 0), ("s_nop 7", 0)):
        assert len(hazards([line.format(nop) for line in code])) == bad
    assert hazards(["<k>:", "s_mov_b32 m0, s4", "global_load_lds_dwordx4 v[0:1], off lds"])
    assert not hazards(["<k>:", "s_mov_b32 m0, s4", "s_nop 0",
                        "global_load_lds_dwordx4 v[0:1], off lds"])
    assert hazards(["<k>:", "v_cmp_gt_i32_e64 s[4:5], s2, v0", "s_nop 3",
                    "global_load_dword v1, v0, s[4:5]"])


def test_waits_before_memory_instructions(tmp_path):
    loads, found = 0, []
    for name, lines in instructions(tmp_path):
        loads += sum("buffer_load_dwordx4" in x and " lds" in x for x in lines)
        found += hazards(lines)
    assert loads > 1000  # the loads into LDS are among what was read
    assert not found, "\n".join(map(str, found[:20]))
