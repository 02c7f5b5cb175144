"""The attention over selected pages loads its tiles with the same written-out instructions as the attention over whole caches, so the compiled code is held to
the same rule: nothing else uses m0, and five cycles lie between its write and the load.  No GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2605_02218_amd import build as B
from test_isa_attend import stray_m0


@pytest.mark.skipif(not (os.path.exists(B._hipcc()) or shutil.which(B._hipcc())), reason="no hipcc")
def test_only_the_written_out_loads_use_m0(tmp_path):
    out = str(tmp_path / "sparse.s")
    subprocess.run([B._hipcc(), *B.FLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, "sparse.hip"), "-o", out], check=True, stderr=subprocess.PIPE)
    with open(out) as f:
        bad, loads = stray_m0(f.read().split("\n"))
    assert bad == [] and loads > 100
