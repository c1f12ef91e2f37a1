"""What the kernels' sources have to say for a compiler to keep them safe."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_06812_b200", "csrc")
BYTES = {"uint4": 16, "int4": 16, "float4": 16, "double2": 16, "ulonglong2": 16, "uint2": 8, "int2": 8, "float2": 8, "uint64_t": 8}


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu"))), ids=os.path.basename)
def test_shared_arrays_read_by_vectors_are_aligned_for_them(path):
    """An array of small elements in shared memory lies where the compiler puts it: a vector access to it is a fault unless its
    declaration asks for the vector's alignment."""
    text = open(path).read()
    asked = {}
    for align, names in re.findall(r"^\s*__shared__\s+(?:__align__\((\d+)\)\s+)?\w+\s+([^;]*);", text, re.M):
        for name in re.findall(r"(\w+)\s*\[", re.sub(r"\[[^\]]*\]", "[", names)):
            asked[name] = int(align or 1)
    for vector, name in re.findall(r"reinterpret_cast<(?:const\s+)?(\w+)\s*\*>\(&?(\w+)", text):
        if vector in BYTES and name in asked:
            assert asked[name] >= BYTES[vector], f"{name} is accessed by {vector}"
