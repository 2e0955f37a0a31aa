"""Workgroups of the masked attention's kernels to a compute unit, from the
registers and LDS of the compiled kernels (no GPU needed)."""

import os
import re
import subprocess

import pytest

from paper_2412_02962_amd import build

# by blocks of 32 channels
PER_CU = {"masked_forward": {2: 3, 3: 2, 4: 2}, "masked_few": {2: 2, 3: 1, 4: 1}, "masked_dq": {2: 3, 3: 2, 4: 2},
          "masked_dkv": {2: 2, 3: 2, 4: 2}}


@pytest.mark.parametrize("source,kernels", [("masked_forward.hip", ("masked_forward", "masked_few")),
                                            ("masked_backward.hip", ("masked_dq", "masked_dkv"))])
def test_workgroups_of_a_compute_unit(source, kernels):
    src = os.path.join(build.CSRC, source)
    r = subprocess.run([build.hipcc()] + build.flags_of(src) + ["--cuda-device-only", "-S", "-o", "-", src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    seen = set()
    for doc in re.split(r"\n  - \.agpr_count:", r.stdout)[1:]:
        field = lambda f: int(re.search(rf"\.{f}:\s+(\d+)", doc).group(1))
        kind = re.search(r"\.name:\s+_Z\S*?(masked_(?:forward|few|dq|dkv))ILi(\d)E", doc)
        if not kind:
            continue
        threads, regs, lds = field("max_flat_workgroup_size"), field("vgpr_count"), field("group_segment_fixed_size")
        # a SIMD has 512 registers a lane, given out by eight
        fit = min(4 * (512 // (-(-regs // 8) * 8)) * 64 // threads, 160 * 1024 // lds)
        assert fit >= PER_CU[kind[1]][int(kind[2])], (kind[0], regs, lds)
        seen.add((kind[1], int(kind[2])))
    assert seen == {(k, d) for k in kernels for d in (2, 3, 4)}
