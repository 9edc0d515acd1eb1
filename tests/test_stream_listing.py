"""What the compiler made of the norm in few bits, the 4-bit maps and the log probabilities: no register goes to memory, loops whose source asks for it are
unrolled, and the main loop of every 4-bit tile kernel waits for loads into LDS where its source says so and nowhere else.  (Before an LDS read that it cannot
tell from the target of a load the compiler waits for all of them; so it does where it has lost count of a register's load.)"""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2506_06295_amd import build

SOURCES = ("kernels_mx4.hip", "kernels_norm8.hip", "kernels_logprobs.hip")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    to = tmp_path_factory.mktemp("listing")

    def compile_one(src):
        out = to / (src + ".s")
        err = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", str(out)], check=True,
                             capture_output=True, text=True).stderr
        return out.read_text(), err
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(compile_one, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_registers_and_loops(listings, src):
    text, err = listings[src]
    assert "loop not unrolled" not in err
    sizes = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
    assert sizes and set(sizes) == {"0"}
    assert set(re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)) == {"0"}


def loops(text):
    """(kernel, lines) of the shortest loop of every tile kernel that both multiplies and loads into LDS."""
    for name, body in re.findall(r"^(_Z\w*k_mx4_wide\w*):(.*?)^\.Lfunc_end", text, re.S | re.M):
        lines, labels, best = body.splitlines(), {}, None
        for i, line in enumerate(lines):
            m = re.match(r"(\.LBB\w+):", line)
            if m:
                labels[m[1]] = i
            m = re.search(r"s_c?branch\w* (\.LBB\w+)", line)
            if m and m[1] in labels:
                loop = lines[labels[m[1]]:i + 1]
                if any("v_mfma" in x for x in loop) and any("global_load_lds" in x for x in loop) and (best is None or len(loop) < len(best)):
                    best = loop
        yield name, best


def waits(loop):
    return [int(n) for line in loop for n in re.findall(r"vmcnt\((\d+)\)", line)]


def test_main_loops_wait_once(listings):
    found = dict(loops(listings["kernels_mx4.hip"][0]))
    assert len(found) == 14   # seven tiles, two types
    for name, loop in found.items():
        tiles = [int(n) for n in re.search(r"Li(\d)ELi(\d)E", name).groups()]
        assert sum("v_mfma_scale_f32_32x32x64_f8f6f4" in line for line in loop) == 4 * tiles[0] * tiles[1], name
        assert len(waits(loop)) == 1 and waits(loop)[0] > 0, (name, waits(loop))


def test_the_reader_sees_a_wait_too_many(listings):
    name, loop = next(loops(listings["kernels_mx4.hip"][0]))
    at = next(i for i, line in enumerate(loop) if "ds_read" in line)
    assert waits(loop[:at] + ["\ts_waitcnt vmcnt(0)"] + loop[at:]) != waits(loop)
