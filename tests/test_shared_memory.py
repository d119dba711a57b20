"""Arrays in shared memory that are read or written 8 or 16 bytes at a time say that they are so aligned."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_23286_amd", "csrc")
WIDTH = {"float4": 16, "uint4": 16, "int4": 16, "u32x4": 16, "f32x4": 16, "bf16x8": 16, "float2": 8, "uint2": 8, "u32x2": 8,
         "i16x4": 8}


def wide_uses(text):
    """(array, bytes) of casts of an array's own elements to a wider type."""
    for m in re.finditer(r"reinterpret_cast<(?:const )?(\w+) ?\*>\(&?(s_\w+|lds)\b", text):
        if m[1] in WIDTH:
            yield m[2], WIDTH[m[1]]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.hip"))), ids=os.path.basename)
def test_wide_accesses_to_shared_arrays_are_aligned(path):
    text = open(path).read()
    # a kernel's text runs from its __global__ to the next one's
    for kernel in re.split(r"(?=__global__)", text):
        for name, width in wide_uses(kernel):
            for decl in re.findall(r"__shared__[^;]*?\b%s\b[^;]*;" % name, kernel):
                m = re.search(r"aligned\((\d+)\)", decl)
                assert m and int(m[1]) >= width, f"{name} is used {width} bytes at a time: {decl}"
