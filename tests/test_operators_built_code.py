"""What the kernels of the paged cache and of the verification were compiled to: what they keep in registers is in registers, and results of matrix instructions are waited for, also where
they lie in accumulation registers."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2504_08860_amd as H
import test_matrix_instruction_waits as waits
from paper_2504_08860_amd.build import build_library
from test_kernel_registers import OBJDUMP, READELF

KERNELS = r"\dk_(paged|attend|verify)"
MOST = 160   # bytes a lane: many rows of fp32 heads wider than 128 have 33 values too many for their 256 registers, queries in three parts among them


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    at = tmp_path_factory.mktemp("code")
    if not os.path.exists(H.LIB_PATH):
        build_library()
    shutil.copy(H.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    return [str(at / f) for f in sorted(os.listdir(at)) if f.endswith("gfx950")]


@pytest.mark.skipif(READELF is None or OBJDUMP is None, reason="no llvm-readelf")
def test_scratch_memory(code):
    scratch = {}
    for path in code:
        notes = subprocess.run([READELF, "--notes", path], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
            name = re.search(r"\n\s+\.name:\s+(_Z\S+)", kernel)
            if name and re.search(KERNELS, name.group(1)):
                scratch[name.group(1)] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel).group(1))
    assert len(scratch) > 40
    assert not {name: n for name, n in scratch.items() if n > MOST}


def registers_of_both_kinds(operand):
    out = set()
    for kind, first, last, kind_of_one, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", operand):
        out |= {(kind_of_one, int(one))} if one else {(kind, n) for n in range(int(first), int(last) + 1)}
    return out


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_results_in_accumulation_registers_are_waited_for(code, monkeypatch):
    monkeypatch.setattr(waits, "registers", registers_of_both_kinds)
    found, count = [], 0
    for path in code:
        for name, instructions in waits.functions(path):
            if re.search(KERNELS, name):
                n, fault = waits.too_early(instructions)
                count += n
                if fault:
                    found.append((name, fault))
    assert count > 1000
    assert not found, "\n".join(f"{name}: {fault}" for name, fault in found[:5])


def test_what_is_found_there(monkeypatch):
    monkeypatch.setattr(waits, "registers", registers_of_both_kinds)
    code = lambda *lines: [(4 * i, op, rest) for i, (op, rest) in enumerate(lines)]  # noqa: E731
    m, read, end = ("v_mfma_f32_16x16x32_bf16", "a[4:7], v[0:3], v[8:11], a[4:7]"), ("v_accvgpr_read_b32", "v9, a5"), ("s_endpgm", "")
    assert waits.too_early(code(m, read, end))[1] and waits.too_early(code(m, ("s_nop", "6"), read, end))[1]
    assert not waits.too_early(code(m, ("s_nop", "7"), read, end))[1] and not waits.too_early(code(m, ("v_mov_b32_e32", "v5, v6"), end))[1]
