"""Arrays in LDS that store8 writes 16 bytes at a time say so where they are
declared: float alone promises 4 (no GPU needed)."""

import os
import re

import pytest

from paper_2412_02962_amd import build

SOURCES = [os.path.basename(s) for s in build.sources() if "store8(" in open(s).read()]


def unaligned(text):
    """Names of a source's shared arrays that store8 writes and that are declared without aligned(16)."""
    written = set(re.findall(r"store8\((\w+)", text))
    out = []
    for attr, names in re.findall(r"__shared__ (__attribute__\(\(aligned\(16\)\)\) )?float ([^;]*);", text):
        out += [n for n in re.findall(r"(\w+)\[", re.sub(r"\[[^\]]*\]", "[", names)) if n in written and not attr]
    return out


def test_the_check_finds_them():
    text = "__shared__ float a[2 * N], b[M[0]];\n__shared__ __attribute__((aligned(16))) float c[4][8];\nstore8(a + r, v); store8(c[0], v);"
    assert unaligned(text) == ["a"]


@pytest.mark.parametrize("source", SOURCES)
def test_arrays_of_whole_vectors(source):
    assert unaligned(open(os.path.join(build.CSRC, source)).read()) == []
