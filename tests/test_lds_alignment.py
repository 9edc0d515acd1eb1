"""LDS arrays that are read or written sixteen bytes at a time state that alignment: the element type's alone is what the language gives an
array, and what a compiler adds to it today it may leave out tomorrow.  The sources are read, nothing is compiled."""
import os
import re

import pytest

from paper_2506_06295_amd import build

WIDE = {"uint4": 16, "int4": 16, "float4": 16, "f32x4": 16, "i32x4": 16, "bf16x8": 16, "uint2": 8, "float2": 8, "int2": 8}
SOURCES = sorted(f for f in os.listdir(build.CSRC) if f.endswith((".hip", ".hpp")))


def shared_arrays(text):
    """(name, alignment that its declaration states) of every LDS array."""
    for m in re.finditer(r"__shared__\s+(?:__attribute__\(\(aligned\((\d+)\)\)\)\s+)?(\w+)\s+([^;]*);", text):
        for name in re.findall(r"(\w+)\s*(?:\[[^\]]*\])+", m[3]):
            yield name, max(int(m[1] or 0), WIDE.get(m[2], 4))


def too_wide(text):
    """(array, type) of casts of an LDS array to a pointer that asks for more than its declaration states."""
    found = dict(shared_arrays(text))
    return [(name, to) for to, name in re.findall(r"reinterpret_cast<(?:const\s+)?(\w+)\s*\*>\(&?(\w+)", text)
            if found.get(name, 16) < WIDE.get(to, 4)]


@pytest.mark.parametrize("source", SOURCES)
def test_wide_accesses_are_aligned(source):
    with open(os.path.join(build.CSRC, source)) as f:
        assert too_wide(f.read()) == []


def test_the_reader_sees_an_array_of_four_byte_alignment():
    text = "__shared__ int a[64], b[3];\n__shared__ __attribute__((aligned(16))) int c[8];\n__shared__ uint4 d[4];\n"
    uses = "reinterpret_cast<const int4*>({0})[i]; reinterpret_cast<uint4*>(&{0}[4]);"
    assert too_wide(text + uses.format("a")) == [("a", "int4"), ("a", "uint4")]
    assert too_wide(text + uses.format("c")) == too_wide(text + uses.format("d")) == []
