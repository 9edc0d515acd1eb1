"""Wait states around the MFMAs that the 8-bit tile kernels write as asm statements: the walk of test_tile_listing over
kernels_i8.hip.  A 16 x 16 x 64 int8 MFMA takes as many passes as the bf16 one of 32, and its result as many wait states: the listing's
own builtin products are held to the same distances."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_06295_amd import build
from tests.test_tile_listing import faults, registers


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("listing") / "kernels_i8.s"
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "kernels_i8.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    found, name = {}, None
    for line in out.read_text().splitlines():
        m = re.match(r"(_Z\w*k_i8_wide\w*):", line)
        if m:
            name = m[1]
            found[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name:
            found[name].append(line)
    return found


def test_no_access_comes_too_early(kernels):
    assert len(kernels) == 14   # seven tiles, two types
    for name, lines in kernels.items():
        assert sum("v_mfma_i32_16x16x64_i8" in l for l in lines) >= 16, name
        assert faults(lines) == [], name


def test_the_walk_finds_a_move_between_the_mfmas(kernels):
    for name, lines in kernels.items():
        at = [i for i, l in enumerate(lines) if "v_mfma" in l]
        dst = registers(lines[at[-1]].split(",")[0])[0][1]
        assert faults(lines[:at[-1] + 1] + [f"\tv_accvgpr_read_b32 v0, a{dst}"] + lines[at[-1] + 1:]), name
