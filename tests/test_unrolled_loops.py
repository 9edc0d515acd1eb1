"""Loops whose source asks to be unrolled are: a pragma that the compiler could not follow says something about the code that is not so."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2506_06295_amd import build

SOURCES = ("kernels_attn_kv4.hip", "kernels_evict.hip", "kernels_i8.hip", "kernels_kv4.hip", "kernels_weigh.hip")


@pytest.fixture(scope="module")
def warnings():
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")

    def compile_one(src):
        return subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", os.devnull],
                              check=True, capture_output=True, text=True).stderr
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(compile_one, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_no_loop_stays_rolled_against_its_pragma(warnings, src):
    assert "loop not unrolled" not in warnings[src]
