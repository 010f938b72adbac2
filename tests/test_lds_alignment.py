"""Arrays in LDS that the layers for several kinds of rows read or write by pieces of 8 or 16 bytes are declared so aligned, in the sources: an array of floats
promises four bytes, whatever a compiler makes of it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_09887_amd", "csrc")
SOURCES = [f for k in ("group_*.hip", "grouped_*", "dropout.hip") for f in sorted(glob.glob(os.path.join(CSRC, k)))]
BYTES = {"float": 4, "int": 4, "int32_t": 4, "uint16_t": 2, "int64_t": 8, "float2": 8, "uint2": 8, "float4": 16, "uint4": 16}


def misdeclared(text):
    """(name, declared alignment, bytes of a piece) of arrays in LDS whose declaration promises less than a piece that they are taken in"""
    wrong, declared = [], {}
    for m in re.finditer(r"__shared__ (?:__attribute__\(\(aligned\((\d+)\)\)\) )?(\w+) (\w+)\[|reinterpret_cast<(?:const )?(\w+) \*>\(&(\w+)\[", text):
        if m.group(3):
            declared[m.group(3)] = max(int(m.group(1) or 0), BYTES[m.group(2)])
        elif m.group(5) in declared and declared[m.group(5)] < BYTES.get(m.group(4), 0):      # (a template's type: no piece)
            wrong.append((m.group(5), declared[m.group(5)], BYTES[m.group(4)]))
    return wrong


def test_a_planted_one_is_seen():
    use = "*reinterpret_cast<const float4 *>(&zs[r][4 * q])"
    assert misdeclared("__shared__ float zs[8][128];" + use) == [("zs", 4, 16)]
    assert not misdeclared("__shared__ __attribute__((aligned(16))) float zs[8][128];" + use)


@pytest.mark.parametrize("source", SOURCES, ids=os.path.basename)
def test_declarations(source):
    assert not misdeclared(open(source).read())
