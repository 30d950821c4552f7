"""What the operators' kernels keep in registers is in registers: how much of it the compiler has put into memory, a lane, as the built library says itself."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2504_08860_amd as H
from paper_2504_08860_amd.build import build_library

READELF, OBJDUMP = (next((p for p in (f"/opt/rocm/llvm/bin/{n}", shutil.which(n) or "") if os.path.exists(p)), None) for n in ("llvm-readelf", "llvm-objdump"))
MOST = 128   # bytes; kernels that have a few values too many for their registers are not split for them


@pytest.mark.skipif(READELF is None or OBJDUMP is None, reason="no llvm-readelf")
@pytest.mark.parametrize("kernels", ["norm", "logprobs", "q4"])
def test_scratch_memory(kernels, tmp_path):
    library = tmp_path / "lib.so"
    if not os.path.exists(H.LIB_PATH):
        build_library()
    shutil.copy(H.LIB_PATH, library)
    subprocess.run([OBJDUMP, "--offloading", str(library)], cwd=tmp_path, check=True, capture_output=True)
    scratch = {}
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950"):
            notes = subprocess.run([READELF, "--notes", str(tmp_path / f)], check=True, capture_output=True, text=True).stdout
            for kernel in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
                name = re.search(r"\n\s+\.name:\s+(_Z\S+)", kernel)
                if name and re.search(rf"\dk_\w*{kernels}", name.group(1)):
                    scratch[name.group(1)] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel).group(1))
    assert len(scratch) > 10
    assert not {name: n for name, n in scratch.items() if n > MOST}
