"""The ctypes mirrors of the operators' structs have the C compiler's sizes and offsets, and their constants the header's values."""
import ctypes
import os
import subprocess

import paper_2504_08860_amd as H

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layout_and_constants_match_the_header(tmp_path):
    structs = {"hbp_q4_matrix_t": H.hbp_q4_matrix_t, "hbp_norms_t": H.hbp_norms_t}
    constants = {"HBP_F32": 0, "HBP_F16": 1, "HBP_BF16": 2, "HBP_GATE_NONE": H.operators.GATE_NONE, "HBP_GATE_CHANNEL": H.operators.GATE_CHANNEL,
                 "HBP_GATE_TOKEN": H.operators.GATE_TOKEN, "HBP_GATE_FULL": H.operators.GATE_FULL}
    asked, want = [], []
    for name, mirror in structs.items():
        asked.append(f"(long)sizeof({name})")
        want.append(ctypes.sizeof(mirror))
        for field, _ in mirror._fields_:
            asked.append(f"(long)offsetof({name}, {field})")
            want.append(getattr(mirror, field).offset)
    for name, value in constants.items():
        asked.append(f"(long){name}")
        want.append(value)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hbp.h"\nint main(void){' + "".join(f'printf("%ld\\n", {a});' for a in asked) + "return 0;}")
    subprocess.check_call(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    assert [int(v) for v in subprocess.check_output([str(tmp_path / "layout")]).split()] == want


def test_shapes_of_a_4_bit_matrix():
    assert H.hbp_q4_shapes(3, 1, 32) == ((3, 16), (3, 1))
    assert H.hbp_q4_shapes(5, 33, 32) == ((5, 32), (5, 2))
    assert H.hbp_q4_shapes(5, 4096) == ((5, 2048), (5, 32))
