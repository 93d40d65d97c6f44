"""Loads from global memory straight into LDS take their base from M0, and a scalar instruction's write of M0 needs one wait
state before them. They are inline assembly, for which the compiler places no waits: the built library is looked at (its own
kernels' code, no GPU).
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_22533_amd import f3c

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"



@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_a_wait_state_between_m0_and_the_load(tmp_path):
    f3c.lib()
    shutil.copy(f3c.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    loads, early = 0, []
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" not in name:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", name], cwd=tmp_path, check=True,
                              capture_output=True, text=True).stdout
        kernel = before = ""
        for line in text.splitlines():
            if m := re.match(r"(?:[0-9a-f]+ )?<(\w+)>:", line):
                kernel, before = m.group(1), ""
                continue
            line = line.split("//")[0].strip()
            if not line:
                continue
            if re.match(r"buffer_load\w* .*\blds\b|global_load_lds", line):
                loads += 1
                if re.match(r"s_\w+ m0\b", before):
                    early.append((kernel, before, line))
            before = line
    assert loads > 3000
    assert not early, (len(early), loads, early[:3])
