"""The gfx950 code of the linear layers as built here (no GPU).  A step of
their loop ends with a barrier that leaves the wave's last LDS reads open; it
holds only if no LDS store lies among those, which is a property of the
instructions' final order."""
import os
import re

import pytest

from paper_2606_11081_amd import build as lib_build
from tests.test_build_isa import BUNDLER, OBJDUMP, _disassemble


@pytest.mark.skipif(not (os.path.exists(BUNDLER) and os.path.exists(OBJDUMP)), reason="ROCm LLVM tools absent")
def test_steps_wait_for_their_lds_stores(tmp_path):
    text = _disassemble("linear.hip", tmp_path)
    kernels = [b for b in re.split(r"\n(?=[0-9a-f]{16} <)", text) if "k_linearI" in b.split("\n")[0]]
    assert kernels
    checked = 0
    for body in kernels:
        lines = [re.sub(r"\s*//.*", "", l).strip() for l in body.split("\n")]
        for at, line in enumerate(lines):
            wait = re.match(r"s_waitcnt lgkmcnt\((\d+)\)$", line)
            if not (wait and lines[at + 1] == "s_barrier"):
                continue
            after = 0
            for earlier in reversed(lines[:at]):
                if earlier.startswith("ds_write") or earlier == "s_barrier":
                    break
                after += earlier.startswith("ds_")
            assert int(wait.group(1)) <= after, (lines[0], at, line, after)
            checked += 1
    assert checked >= 4 * len(kernels)
    assert "linear.hip" in lib_build.EXTRA
