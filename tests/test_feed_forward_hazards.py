"""A memory instruction may read a scalar register five wait states after a
vector instruction wrote it, not sooner.  The compiler does not look into inline
assembly, so the compiled loads of the feed-forward products are looked at here
(no GPU needed)."""

import os
import re
import subprocess

import pytest

from paper_2412_02962_amd import build

WAIT_STATES = 5
WRITERS = ("v_readfirstlane", "v_readlane", "v_cmp")
READERS = ("buffer_", "global_", "flat_", "scratch_")


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if not m:
        return {operand} if operand == "m0" else set()
    first, last = (m[1], m[2]) if m[1] else (m[3], m[3])
    return {f"s{i}" for i in range(int(first), int(last) + 1)}


def early_reads(assembly):
    """The memory instructions that read a scalar register too early."""
    since, found = {}, []  # register -> wait states since its vector write
    for line in assembly.splitlines():
        t = line.split(";")[0].replace(",", " ").split()
        if not t or t[0].startswith(".") or t[0].endswith(":"):
            continue
        if t[0].startswith(READERS):
            read = set().union(*map(_scalars, t[1:])) | ({"m0"} if "lds" in t[1:] else set())
            found += [line.strip() for r in read if since.get(r, WAIT_STATES) < WAIT_STATES]
        states = int(t[1]) + 1 if t[0] == "s_nop" else 1
        since = {r: n + states for r, n in since.items() if n + states < WAIT_STATES}
        if t[0].startswith(WRITERS):
            since.update(dict.fromkeys(_scalars(t[1]), 0))
        elif t[0].startswith("s_") and len(t) > 1:
            for r in _scalars(t[1]):
                since.pop(r, None)
    return found


@pytest.mark.parametrize("wait,early", [("s_nop 3", 1), ("s_nop 4", 0), ("s_mov_b32 s6, s9", 0)])
def test_the_reader_of_assembly(wait, early):
    code = f"\tv_readfirstlane_b32 s6, v1\n\t{wait}\n\tbuffer_load_dwordx4 v2, s[4:7], 0 offen lds\n"
    assert len(early_reads(code)) == early


def test_no_load_reads_its_buffer_too_early():
    src = os.path.join(build.CSRC, "ff_product.hip")
    r = subprocess.run([build.hipcc()] + build.flags_of(src) + ["--cuda-device-only", "-S", "-o", "-", src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert "offen lds" in r.stdout
    assert early_reads(r.stdout) == []
