"""Values at the ends of the types' ranges in the feed-forward sub-layer's
operators."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, F64, BF16 = "cuda", torch.float64, torch.bfloat16


@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 130])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("last", [2.0 ** 58, 2.0 ** 58 * (1 - 2.0 ** -6)])
def test_an_infinite_h(M, kind, last):
    """v and g are 63 * 2^58 + last: 2^64, whose h = 2^128 is infinite, or 2^64 -
    2^52, whose h is finite in float32 and infinite in bf16.  Positive weights
    give an infinite y, whatever way h takes between the products."""
    from paper_2412_02962_amd import pcpp
    print("[case] infinite h", M, kind, last, flush=True)
    C, F = 64, 128
    w1 = torch.full((2 * F, C), 2.0 ** 58)
    w1[:, 5] = last
    w = dict(ff1_w=w1, ff1_b=None, ff2_w=torch.ones(C, F), ff2_b=None)
    w = {k: None if v is None else v.to(DEV, BF16) for k, v in w.items()}
    x = torch.ones(M, C, device=DEV, dtype=BF16)
    y = torch.zeros(M, C, device=DEV, dtype=BF16)
    g = pcpp.make_ff_geom(M, C, F, pcpp.PCPP_ACT_SILU if kind == "silu" else pcpp.PCPP_ACT_GELU)
    n = pcpp.pcpp_gated_ff_workspace_size(g)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    pcpp.pcpp_gated_ff(g, pcpp.make_ff_weights(w), x, y, None, None, ws, n)
    torch.cuda.synchronize()
    assert bool((y == float("inf")).all()), y[0, :4]
