"""Register spills of the kernels that multiply narrow operands, from the metadata the compiler leaves in the objects of the last build
(nothing to look at where only the linked library is there)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LLVM = "/opt/rocm/llvm/bin"
BUILD = os.path.join(ROOT, "paper_2605_14929_amd", "csrc", "_build")
UNITS = ("f8", "f8mm", "wgrad", "packed")


def _object(unit):
    return os.path.join(BUILD, unit + ".o")


@pytest.mark.skipif(not all(os.path.exists(_object(u)) for u in UNITS) or not shutil.which(f"{LLVM}/clang-offload-bundler"), reason="no objects of a build, or no tools to read them")
@pytest.mark.parametrize("unit", UNITS)
def test_no_kernel_spills(unit, tmp_path):
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.check_call([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", _object(unit), str(tmp_path / "copy")], stderr=subprocess.DEVNULL)
    subprocess.check_call([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={code}"])
    notes = subprocess.run([f"{LLVM}/llvm-readobj", "--notes", code], capture_output=True, text=True, check=True).stdout
    seen = 0
    for part in re.split(r"\n\s+- \.a", notes)[1:]:
        f = dict(re.findall(r"\.?(\w+):\s+(\S+)", part))
        if "symbol" not in f:
            continue
        seen += 1
        assert int(f["vgpr_spill_count"]) == 0 and int(f["sgpr_spill_count"]) == 0, f["symbol"]
        assert int(f["group_segment_fixed_size"]) <= 160 * 1024, f["symbol"]
    assert seen >= 8
