"""Signalling NaN in the feed-forward sub-layer's operators."""

import pytest
import torch

from tests import ff_reference as ref

pytestmark = pytest.mark.gpu
DEV, BF16, U8 = "cuda", torch.bfloat16, torch.uint8


def _say(*a):
    print("[case]", *a, flush=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_signalling_nan_leaves_its_group_as_it_is(dtype):
    """Every pair of a NaN's place and that of the group's largest value among
    eight channels: codes and scale are those of the finite values."""
    from paper_2412_02962_amd import pcpp
    _say("signalling nan", dtype)
    pairs = [(i, j) for i in range(8) for j in range(8) if i != j]
    gen = torch.Generator().manual_seed(4)
    x = torch.rand((len(pairs), 32), generator=gen) + 0.5
    for r, (_, big) in enumerate(pairs):
        x[r, 8 + big] = 1000.0
    if dtype == "f32":
        bits = x.view(torch.int32)
        for r, (nan, _) in enumerate(pairs):
            bits[r, 8 + nan] = 0x7f800001 if r % 2 else -0x7fffff  # 0xff800001
        code = pcpp.PCPP_DTYPE_F32
    else:
        x = x.to(BF16)
        bits = x.view(torch.int16)
        for r, (nan, _) in enumerate(pairs):
            bits[r, 8 + nan] = 0x7f81 if r % 2 else -0x7f  # 0xff81
        code = pcpp.PCPP_DTYPE_BF16
    assert int(x.isnan().sum()) == len(pairs)
    codes, scales = torch.zeros(x.shape, dtype=U8, device=DEV), torch.zeros((len(pairs), 1), dtype=U8, device=DEV)
    pcpp.pcpp_checkpoint_save(len(pairs), 32, code, x.to(DEV), codes, scales)
    torch.cuda.synchronize()
    want_c, want_s = ref.to_8bit(x)
    got, nan = codes.cpu(), (want_c & 127) == 127
    assert torch.equal(scales.cpu(), want_s)
    assert ((got & 127) == 127)[nan].all() and torch.equal(got[~nan], want_c[~nan])
