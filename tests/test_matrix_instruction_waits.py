"""The built library's matrix instructions are left the time they take.

A 16x16x32 matrix instruction takes four passes and gfx950 does not wait by itself for its results: between it and a vector instruction that reads or writes one of its result registers, a store
of one, or a matrix instruction that multiplies one, the compiler has to leave eight wait states (passes + 4; an instruction is one, s_nop n is n + 1).  It does so in straight-line code, but behind a
conditional branch it has been seen to leave one, with wrong results.  So the code is read here: along every way of control flow from every matrix instruction."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2504_08860_amd as H
from paper_2504_08860_amd.build import build_library

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump") or "") if os.path.exists(p)), None)
STATES = 8
LOADS = ("ds_read", "ds_bpermute", "global_load", "buffer_load", "flat_load", "scratch_load")   # (their first operand is written when the data come)


def registers(operand):
    out = set()
    for first, last, one in re.findall(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", operand):
        out |= {int(one)} if one else set(range(int(first), int(last) + 1))
    return out


def functions(path):
    """(name, [(address, instruction, operands)]) of those with matrix instructions"""
    name, code, matrix = None, [], False
    with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", path], stdout=subprocess.PIPE, text=True) as dump:
        for line in dump.stdout:
            if line.startswith("\t") and "//" in line:
                text, _, address = line.partition("//")
                op, _, rest = text.strip().partition(" ")
                code.append((int(address.split(":")[0], 16), op, rest))
                matrix |= op.startswith("v_mfma")
            elif line.rstrip().endswith(">:"):
                if matrix:
                    yield name, code
                name, code, matrix = line.split("<")[1].split(">")[0], [], False
        if matrix:
            yield name, code
    assert dump.returncode == 0


def too_early(code):
    place = {address: i for i, (address, _, _) in enumerate(code)}
    operands = [[o.strip() for o in re.split(r",\s*(?![^\[]*\])", rest)] for _, _, rest in code]
    count = 0
    for i, (_, op, _) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        assert "_16x16x32_" in op, f"{op}: how long it takes is not known here"
        count += 1
        result, ways, seen = registers(operands[i][0]), [(i + 1, 0)], {}
        while ways:
            at, states = ways.pop()
            while at < len(code) and states < STATES and seen.get(at, STATES) > states:
                seen[at] = states
                address, op, _ = code[at]
                if op == "s_endpgm":
                    break
                if op.startswith("v_mfma"):
                    if (registers(operands[at][1]) | registers(operands[at][2])) & result:
                        return count, (code[i], code[at], states)
                    if registers(operands[at][0]) & result:      # (goes on with the sum: a shorter wait, between matrix instructions, and the results are that one's from here on)
                        break
                elif not op.startswith("s_") and any(registers(o) & result for o in operands[at][1 if op.startswith(LOADS) else 0:]):
                    return count, (code[i], code[at], states)
                if op.startswith(("s_cbranch", "s_branch")):
                    jump = int(operands[at][0].split()[0])
                    ways.append((place[address + 4 + 4 * (jump - 65536 if jump > 32767 else jump)], states + 1))
                    if op == "s_branch":
                        break
                states += int(operands[at][0].split()[0], 0) + 1 if op == "s_nop" else 1
                at += 1
    return count, None


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_nothing_touches_the_results_of_a_matrix_instruction_too_early(tmp_path):
    library = tmp_path / "lib.so"
    if not os.path.exists(H.LIB_PATH):
        build_library()
    shutil.copy(H.LIB_PATH, library)
    subprocess.run([OBJDUMP, "--offloading", str(library)], cwd=tmp_path, check=True, capture_output=True)
    found, count = [], 0
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950"):
            for name, code in functions(str(tmp_path / f)):
                n, fault = too_early(code)
                count += n
                if fault:
                    found.append((name, fault))
    assert count > 1000      # (they are found at all)
    assert not found, "\n".join(f"{name}: {writes[1]} {writes[2]} ... {touches[1]} {touches[2]} after {states} wait states" for name, (writes, touches, states) in found)


def test_what_is_found():
    mfma = "v[4:7], v[0:3], v[8:11], v[4:7]"
    code = lambda *lines: [(4 * i, op, rest) for i, (op, rest) in enumerate(lines)]  # noqa: E731
    read, other = ("v_add_f32_e32", "v9, v5, v9"), ("v_add_f32_e32", "v19, v12, v19")
    m = ("v_mfma_f32_16x16x32_bf16", mfma)
    assert too_early(code(m, read, ("s_endpgm", "")))[1]
    assert too_early(code(m, *[other] * 7, read))[1] and not too_early(code(m, *[other] * 8, read))[1]
    assert too_early(code(m, ("s_nop", "6"), read))[1] and not too_early(code(m, ("s_nop", "7"), read))[1]
    assert not too_early(code(m, ("s_endpgm", ""), read))[1]
    assert too_early(code(read, m, ("s_cbranch_vccz", "65533"), ("s_endpgm", "")))[1]               # back to the first
    assert too_early(code(m, ("s_branch", "1"), other, read))[1]                                     # over one
    assert not too_early(code(m, ("ds_read_b128", "v[4:7], v0"), ("s_endpgm", "")))[1] and too_early(code(m, ("ds_read_b128", "v[20:23], v4"), ("s_endpgm", "")))[1]
    assert too_early(code(m, ("v_mfma_f32_16x16x32_bf16", "v[20:23], v[4:7], v[8:11], 0"), ("s_endpgm", "")))[1] and not too_early(code(m, m, ("s_endpgm", "")))[1]
