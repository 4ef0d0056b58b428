"""Shared arrays that a kernel reads as vectors are declared with the vectors' alignment: an array of floats is
guaranteed four bytes, and where the compiler places it may change with any other declaration."""
import glob
import os
import re

import pytest

from paper_2404_14469_b200 import build

BYTES = {"float2": 8, "uint2": 8, "int2": 8, "float4": 16, "uint4": 16, "int4": 16}


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*.cu*"))), ids=os.path.basename)
def test_vector_accesses_of_shared_arrays_are_aligned(path):
    text = re.sub(r"//[^\n]*", "", open(path).read())
    declared = {}
    for attributes, names in re.findall(r"(?<!extern )__shared__ ((?:__align__\(\d+\) )?)\w[\w ]* (\w+\[[^;]*);", text):
        m = re.search(r"\d+", attributes)
        for name in re.findall(r"(\w+)(?:\[[^\]]*\])+", names):
            declared[name] = int(m.group()) if m else 4
    for vector, name in re.findall(r"reinterpret_cast<(?:const )?(\w+)\*>\(&(\w+)\[", text):
        if vector in BYTES and name in declared:
            assert declared[name] >= BYTES[vector], (name, vector)


def test_it_sees_the_arrays_of_the_append_kernel():
    text = open(os.path.join(build.CSRC, "snapkv_append.cu")).read()
    assert len(re.findall(r"reinterpret_cast<const float4\*>\(&(?:cs|sn)\[", text)) == 2
