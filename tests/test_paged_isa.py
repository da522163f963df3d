"""Host-side check of the generated gfx950 code of the paged cache's kernels (no GPU needed; compiles to assembly)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_15601_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _kernels(unit, outdir):
    """Kernel name -> its instructions."""
    from paper_2508_15601_amd import build
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not available")
    out = os.path.join(outdir, unit + ".s")
    subprocess.run([HIPCC, *build.FLAGS, *build.EXTRA.get(unit + ".hip", []), "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only",
                    os.path.join(CSRC, unit + ".hip"), "-o", out], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    found = re.findall(r"^(_ZN4tmw4\S+):\s*;[^\n]*\n(.*?)^\.Lfunc_end", open(out).read(), re.S | re.M)
    return {name: [t for t in (line.strip() for line in body.splitlines()) if t and t[0] not in ";."] for name, body in found}


def test_rope_may_work_in_place(tmp_path):
    """X and Y of tm_rope_apply may be the same memory: neither may be promised to be the only way to it."""
    from paper_2508_15601_amd import build
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "rope.ll")
    subprocess.run([HIPCC, *build.FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "-emit-llvm", "--cuda-device-only", os.path.join(CSRC, "tm_rope.hip"), "-o", out],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    arguments = re.search(r"^define [^\n]*rope_kernel[^(\n]*\((.*)$", open(out).read(), re.M).group(1)
    pointers = re.findall(r"ptr addrspace\(1\)([^%]*)%(\d+|\w+)", arguments)
    X, positions, Y = (pointers[i][0] for i in range(3))
    assert "noalias" in positions and "noalias" not in X and "noalias" not in Y, arguments


def test_pieces_are_planned_in_one_place(tmp_path):
    """How long the pieces of contexts are is worked out in fp32 (with a rounding up that nothing else here has).  Two kernels go by it, and if each worked it out their code would have
    to be alike to the last rounding; so the kernel that puts the pieces together reads what the other left."""
    kernels = _kernels("tm_paged_rows", str(tmp_path))
    plans = {name: any(t.startswith("v_ceil_f32") for t in code) for name, code in kernels.items()}
    merges = [name for name in plans if "paged_rows_merge_kernel" in name]
    rows = [name for name in plans if "paged_rows_kernel" in name or "paged_mixed_kernel" in name]
    assert len(merges) == 2 and len(rows) == 16, sorted(plans)
    assert all(plans[name] for name in rows) and not any(plans[name] for name in merges), plans
