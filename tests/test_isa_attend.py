"""The loads from the pool into LDS of the attention kernels are written out, so two things about the compiled code are the source's own business:
nothing else uses m0, and five cycles lie between its write and the load (one is needed behind m0, five behind a vector instruction that
wrote the address' scalar registers).  Read from the assembly that the compiler makes of the source; no GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_02218_amd import build as B


def stray_m0(lines):
    """(line numbers of uses of m0 other than `s_mov_b32 m0, ..; s_nop 4; global_load_lds`, number of such loads)."""
    code = [(i, x.split(";")[0].strip()) for i, x in enumerate(lines, 1)]
    code = [(i, x) for i, x in code if x and not x.endswith(":") and not x.startswith(".")]
    bad, loads = [], 0
    for n, (i, x) in enumerate(code):
        if "global_load_lds" in x:
            loads += 1
            before = [y for _, y in code[max(0, n - 2):n]]
            if len(before) < 2 or not before[0].startswith("s_mov_b32 m0,") or before[1] != "s_nop 4":
                bad.append(i)
        elif re.search(r"\bm0\b", x) and not (x.startswith("s_mov_b32 m0,") and [y.split()[0] for _, y in code[n + 1:n + 3]][:1] == ["s_nop"]):
            bad.append(i)
    return bad, loads


def test_the_check_sees_another_use():
    good = ["\ts_mov_b32 m0, s3", "\ts_nop 4", "\tglobal_load_lds_dwordx4 v1, s[2:3]"]
    assert stray_m0(good) == ([], 1)
    assert stray_m0(good[:1] + good[2:])[0]
    assert stray_m0(good + ["\tv_readlane_b32 s1, v2, m0"])[0]
    assert stray_m0(["\ts_mov_b32 m0, s3", "\ts_mov_b32 s4, s5"] + good[1:])[0]


@pytest.mark.skipif(not (os.path.exists(B._hipcc()) or shutil.which(B._hipcc())), reason="no hipcc")
def test_only_the_written_out_loads_use_m0(tmp_path):
    out = str(tmp_path / "attend.s")
    subprocess.run([B._hipcc(), *B.FLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, "attend.hip"), "-o", out], check=True, stderr=subprocess.PIPE)
    with open(out) as f:
        bad, loads = stray_m0(f.read().split("\n"))
    assert bad == [] and loads > 100
