"""CPU check of the paged attention's gfx950 code: only its own loads use the register m0.

They write m0 in inline assembly, where a reserved register cannot be declared as overwritten, so no instruction that the
compiler makes may use it.
"""
import os
import subprocess

import pytest

from paper_2607_21475_amd import build


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("src", ["attend_paged.hip", "attend_paged_tiles.hip"])
def test_only_the_loads_use_m0(src, tmp_path):
    out = str(tmp_path / "kernel.s")
    cmd = [build.HIPCC, *build.FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, src), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    own, inside, others = 0, False, []
    for line in open(out):
        text = line.split(";")[0]
        if "ASMSTART" in line:
            inside = True
        elif "ASMEND" in line:
            inside = False
        elif "m0" in text.replace(",", " ").split():
            own += inside
            if not inside:
                others.append(line)
    assert own > 0 and not others, others[:5]
