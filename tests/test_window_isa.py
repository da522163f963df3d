"""Host-side check of the generated gfx950 code of attention in a window (no GPU needed; compiles to assembly): its kernels keep what they work on in registers."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_15601_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.parametrize("unit, kernels", [("tm_paged_window", 15), ("tm_paged_rows_window", 18)])
def test_nothing_is_spilled(unit, kernels, tmp_path):
    """A loop around a block of codes once made the compiler keep every converted code in front of it: 420 bytes a lane in memory, and the kernel took twice its time."""
    from paper_2508_15601_amd import build
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "unit.s")
    subprocess.run([HIPCC, *build.FLAGS, *build.EXTRA.get(unit + ".hip", []), "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only",
                    os.path.join(CSRC, unit + ".hip"), "-o", out], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    sizes = re.findall(r"\.set (\S+paged_\S+)\.private_seg_size, (\d+)", open(out).read())
    assert len(sizes) == kernels, sizes
    assert all(int(n) <= 16 for _, n in sizes), sizes
