"""How a call of tm_paged_attn or tm_paged_attn_window is divided (paged_form in csrc/tm_paged_rows.hip), as far as the host's rules go.  The function is taken from the source and compiled for
the host, with the compute units of an MI355X; no GPU is needed."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_15601_amd", "csrc")
CUS = 256
MAIN = r"""
#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <cstdio>
PARTS
int main()
{
    int bits, heads, run_log, batch, pages, tokens, window, sinks, q_heads, count, len;
    while (scanf("%d %d %d %d %d %d %d %d %d %d %d", &bits, &heads, &run_log, &batch, &pages, &tokens, &window, &sinks, &q_heads, &count, &len) == 11) {
        PagedPool pool{};
        pool.bits = bits, pool.heads = heads, pool.run_log = run_log;
        PagedSeqs s{};
        s.batch = batch, s.max_pages = pages, s.tokens = tokens, s.cap = pages << (run_log + 5);
        s.window = s.cap;
        if ((int64_t)window + sinks < s.cap) s.window = window, s.sinks = sinks;
        const PagedForm f = paged_form(pool, s, q_heads, count, len, CUS);
        printf("%d %d %d %d %d %d %d %d\n", f.columns, f.column_rows, f.column_ctas, (int)(f.alone || f.together), (int)f.together, f.least_rows, f.row_waves, f.target);
    }
}
"""


def _part(name, pattern):
    return re.search(pattern, open(os.path.join(CSRC, name)).read(), re.S | re.M).group(0) + "\n"


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    parts = [_part("tm_paged_device.h", r"^struct PagedPool \{.*?^\};"), _part("tm_paged_device.h", r"^struct PagedSeqs \{.*?^\};"), _part("tm_paged_host.h", r"^constexpr int kPagedMostCtas.*?$"),
             _part("tm_paged_host.h", r"^constexpr int kPagedMostWaves.*?$"), _part("tm_paged_host.h", r"^struct PagedForm \{.*?^\};"), _part("tm_paged_rows_impl.h", r"^constexpr int kLeastStages.*?$"),
             _part("tm_attn_rows_impl.h", r"^constexpr int ST = .*?$"), _part("tm_paged_rows.hip", r"^PagedForm paged_form\(.*?^\}")]
    src, exe = (str(tmp_path_factory.mktemp("rule") / n) for n in ("rule.cpp", "rule"))
    open(src, "w").write(MAIN.replace("PARTS", "".join(parts)).replace("CUS", str(CUS)))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fsanitize=float-cast-overflow,float-divide-by-zero", "-fno-sanitize-recover=all", src, "-o", exe], check=True)

    def ask(calls):
        out = subprocess.run([exe], input="\n".join(" ".join(str(int(x)) for x in c) for c in calls), capture_output=True, text=True)
        assert out.returncode == 0, out.stderr
        names = "columns column_rows column_ctas alone together least_rows row_waves target".split()
        return [dict(zip(names, map(int, line.split()))) for line in out.stdout.splitlines()]
    return ask


def _call(batch, tokens, count, past, bits=8, heads=8, q_heads=32, window=2048, sinks=4, run_log=1):
    return bits, heads, run_log, batch, -(-(past + count) // (32 << run_log)), tokens, window, sinks, q_heads, count, past + count


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("decoding, chunk, past, heads, q_heads, window", [(8, 300, 9000, 2, 16, 2048), (23, 57, 9000, 8, 32, 2048), (64, 512, 20000, 8, 32, 4096), (96, 200, 9000, 8, 32, 2048),
                                                                            (1, 100, 9000, 1, 8, 700), (0, 400, 5000, 2, 8, 512)])
def test_rows_without_new_tokens_do_not_decode(form, bits, decoding, chunk, past, heads, q_heads, window):
    """A chunk and decoding sequences are launched alike whether the table has further rows that are not in the call or not: what is beside the longest new tokens is one token a sequence."""
    calls = [_call(rows, decoding + chunk, chunk, past, bits, heads, q_heads, window) for rows in (max(decoding, 1) + 1, decoding + 5, decoding + chunk, 4 * (decoding + chunk), 65535)]
    forms = form(calls)
    assert all(f["together"] and f["row_waves"] for f in forms), forms
    assert all(f == forms[0] for f in forms), forms


@pytest.mark.parametrize("bits, page_runs", [(8, 1), (4, 0), (4, 2)])
@pytest.mark.parametrize("active, window", [(10, 1 << 30), (32, 1 << 30), (32, 2048), (40, 300)])
def test_segments_are_those_of_sequences_with_tokens(form, bits, page_runs, active, window):
    """A decoding step takes the form of its own sequences, not of the table's rows, where more than half of them are not in it."""
    forms = form([_call(rows, active, 1, 8000, bits, window=window, run_log=page_runs) for rows in (active, 2 * active + 1, 300, 5000)])
    assert all(f == forms[0] for f in forms), forms


def test_share_of_columns_is_within_the_chip(form):
    """Calls of any kind, tables with fewer rows and with more than the call has tokens: nothing is divided by zero or leaves its type (the sanitizer would stop it), and beside row tiles the columns
    have at least a sixteenth of the chip and at most eleven."""
    rng = np.random.default_rng(1)
    calls = []
    for _ in range(4000):
        batch, count, past = (int(2 ** rng.uniform(0, e)) for e in (15, 12, 16))
        tokens = int(2 ** rng.uniform(0, 13))
        heads, group = int(rng.choice([1, 2, 4, 8, 16])), int(rng.choice([1, 2, 5, 8, 16, 64]))
        calls.append(_call(batch, tokens, int(rng.choice([0, count])), past, int(rng.choice([8, 4])), heads, heads * group, int(2 ** rng.uniform(0, 15)), int(rng.choice([0, 4, 200])), int(rng.integers(0, 4))))
    forms = form(calls)
    assert len(forms) == len(calls)
    mixed = [f for f in forms if f["together"]]
    assert len(mixed) > 500 and all(CUS // 16 <= f["column_ctas"] <= CUS * 11 // 16 for f in mixed)


def test_a_window_is_told_from_the_full_call(form):
    """512 tokens after 30000: a window of 4096 is cut otherwise than the whole context; one that reaches as far as the table is no window."""
    full, wide, window = form([_call(1, 512, 512, 30000, window=w, sinks=0) for w in (1 << 30, 30528, 4096)])
    assert full == wide and full["row_waves"] == 8 and full["target"] == CUS
    assert form([_call(8, 16000, 2000, 0, window=256, sinks=0)])[0]["target"] == 0 and window["row_waves"] == 8


def test_hooks_refuse_before_they_look_at_a_device():
    import ctypes
    import paper_2508_15601_amd as tm
    lib = tm.load_library()
    for hook, outs in ((lib.tm_get_paged_window_plan, 4), (lib.tm_get_paged_window_form, 3)):
        assert hook(None, ctypes.c_void_p(4096), 8, 100, 4, *[None] * outs) == -1 and "cache" in tm.tm_last_error()
