"""Host-side check of the generated gfx950 code of attention in a window (no GPU needed; compiles to assembly): not a byte of a lane's memory, which test_window_isa.py allows sixteen of."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_15601_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.parametrize("unit", ["tm_paged_window", "tm_paged_rows_window"])
def test_no_memory_of_a_lane(unit, tmp_path):
    from paper_2508_15601_amd import build
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "unit.s")
    subprocess.run([HIPCC, *build.FLAGS, *build.EXTRA.get(unit + ".hip", []), "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only",
                    os.path.join(CSRC, unit + ".hip"), "-o", out], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    text = open(out).read()
    kernels = re.findall(r"^\s*\.amdhsa_kernel (\S+)", text, re.M)
    sizes = dict(re.findall(r"^\s*\.set (\S+)\.private_seg_size, (\d+)", text, re.M))
    assert kernels and all(sizes.get(k) == "0" for k in kernels), sizes
