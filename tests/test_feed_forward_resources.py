"""Workgroups per compute unit that the feed-forward products' plans count on,
from the registers and LDS of the compiled kernels (no GPU needed)."""

import os
import re
import subprocess

from paper_2412_02962_amd import build

PER_CU = {"0": 2, "1": 2, "2": 1, "3": 3}  # 64 x 128, 128 x 256, 256 x 256 tiles, 64 x 128 in two stages


def test_products_fit_a_compute_unit():
    src = os.path.join(build.CSRC, "ff_product.hip")
    r = subprocess.run([build.hipcc()] + build.flags_of(src) + ["--cuda-device-only", "-S", "-o", "-", src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    seen = set()
    for doc in re.split(r"\n  - \.agpr_count:", r.stdout)[1:]:
        field = lambda f: int(re.search(rf"\.{f}:\s+(\d+)", doc).group(1))
        kind = re.search(r"\.name:\s+_Z\S*ff_(?:products?|gate_grad)ILi(\d)E", doc)
        if not kind:
            continue
        threads, regs, lds = field("max_flat_workgroup_size"), field("vgpr_count"), field("group_segment_fixed_size")
        # vgpr_count is of both files: a SIMD has 512 registers a lane, given out by eight
        fit = min(4 * (512 // (-(-regs // 8) * 8)) * 64 // threads, 160 * 1024 // lds)
        assert fit >= PER_CU[kind.group(1)], (kind.group(0), regs, lds)
        seen.add(kind.group(1))
    assert seen == set(PER_CU)
