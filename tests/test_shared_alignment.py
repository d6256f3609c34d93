"""Shared arrays that kernels read through a wider type say so where they are declared: their place beside other arrays is the compiler's."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_16477_b200", "csrc")
SIZES = {"char": 1, "int8_t": 1, "uint8_t": 1, "bf16": 2, "uint16_t": 2, "int": 4, "unsigned": 4, "uint32_t": 4, "float": 4,
         "double": 8, "long long": 8, "uint64_t": 8, "int64_t": 8, "uint2": 8, "int2": 8, "float2": 8, "uint4": 16, "int4": 16, "float4": 16}
DECLARED = re.compile(r"__shared__\s+(?:(?:__align__|alignas)\((\d+)\)\s+)?((?:unsigned char|unsigned int|long long|\w+))\s+([^;]+);")
WIDER = re.compile(r"reinterpret_cast<(?:const )?(uint2|uint4|int2|int4|float2|float4) \*>\(&?(\w+)")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_shared_arrays_read_through_a_wider_type_are_aligned_for_it(path):
    with open(path) as f:
        text = f.read()
    declared = []      # (place, name, alignment)
    for m in DECLARED.finditer(text):
        own = SIZES.get(m[2].replace("unsigned char", "char").replace("unsigned int", "unsigned"), 1)
        for name in re.findall(r"(\w+)\s*\[", re.sub(r"\[[^\]]*\]", "[]", m[3])):
            declared.append((m.start(), name, max(int(m[1] or 0), own)))
    for m in WIDER.finditer(text):
        before = [d for d in declared if d[1] == m[2] and d[0] < m.start()]
        if before:
            assert before[-1][2] >= SIZES[m[1]], f"{m[2]} is read as {m[1]} (line {text.count(chr(10), 0, m.start()) + 1})"
