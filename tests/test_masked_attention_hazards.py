"""The masked attention's loads straight into LDS, compiled: none reads a scalar
register that a vector instruction wrote less than five wait states before, on
any path (no GPU needed)."""

import os
import subprocess

import pytest

from paper_2412_02962_amd import build
from tests.test_feed_forward_hazard_paths import early_reads


@pytest.mark.parametrize("source", ["masked_forward.hip", "masked_backward.hip"])
def test_no_path_reads_an_address_too_early(source):
    src = os.path.join(build.CSRC, source)
    r = subprocess.run([build.hipcc()] + build.flags_of(src) + ["--cuda-device-only", "-S", "-o", "-", src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert len([line for line in r.stdout.splitlines() if "global_load_lds" in line]) > 100
    assert early_reads(r.stdout) == []
