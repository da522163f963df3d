"""A frequency as a fraction of a turn (rope_turn in csrc/tm_w4_api.hip) against rational arithmetic.  The function is taken from the source and compiled for the host.

96 bits are right to half a unit, and pi is known here to 49 decimals: what is off is off by rounding alone, which for a half is either way."""
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import oracle_paged as op

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_15601_amd", "csrc")
MAIN = r"""
#include <cmath>
#include <cstdint>
#include <cstdio>
using namespace std;
STRUCT
FUNCTION
int main()
{
    double f;
    while (scanf("%la", &f) == 1) {
        const RopeTurn t = rope_turn(f);
        printf("%llu %u\n", (unsigned long long)t.high, t.low);
    }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_turns_are_the_nearest_of_96_bits(tmp_path):
    struct = re.search(r"struct RopeTurn \{.*?\n\};\n", open(os.path.join(CSRC, "tm_rope_device.h")).read(), re.S).group(0)
    function = re.search(r"static RopeTurn rope_turn\(double f\)\n\{.*?\n\}\n", open(os.path.join(CSRC, "tm_w4_api.hip")).read(), re.S).group(0)
    src, exe = tmp_path / "turns.cpp", tmp_path / "turns"
    src.write_text(MAIN.replace("STRUCT", struct).replace("FUNCTION", function))
    subprocess.run(["g++", "-O2", "-std=gnu++17", "-Wall", "-Werror", str(src), "-o", str(exe)], check=True)
    rng = np.random.default_rng(0)
    f = [0.0, 1.0, -1.0, 1e6, -1e6, np.nextafter(1e6, 0), 2 * math.pi, -2 * math.pi, math.pi, 1e-30, 1e-300, 5e-324, -5e-324, 2.0 ** -62, 2.0 ** -63, 2.0 ** -64, 2.0 ** -93, 2.0 ** -96]
    f += [float(10000.0 ** (-2.0 * i / 256)) for i in range(128)]
    f += (np.exp(rng.uniform(math.log(1e-40), math.log(1e6), 4000)) * rng.choice([-1, 1], 4000)).tolist()
    done = subprocess.run([str(exe)], input="\n".join(float(x).hex() for x in f), stdout=subprocess.PIPE, text=True, check=True)
    lines = done.stdout.split("\n")[:-1]
    assert len(lines) == len(f)
    for x, line in zip(f, lines):
        high, low = map(int, line.split())
        off = (op.Fraction(x) / op._TWO_PI * 2 ** 96 - ((high << 32) + low)) % 2 ** 96
        assert min(off, 2 ** 96 - off) <= op.Fraction(1, 2) + op.Fraction(1, 10 ** 6), (x, line)
