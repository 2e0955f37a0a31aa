"""Values at the ends of the types' ranges in the feed-forward sub-layer's
operators."""

import pytest
import torch

from tests import ff_reference as ref

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


@pytest.mark.parametrize("R,C", [(3, 64), (300, 1280), (2, 4096)])
@pytest.mark.parametrize("eps", [1e-30, 1e-37])
def test_the_norm_of_small_rows(R, C, eps):
    """Rows whose rstd, but not its cube, is a float32.  The parts that cancel
    each carry a few float32 roundings: 2^-18 of their size."""
    from paper_2412_02962_amd import pcpp
    print("[case] small rows", R, C, eps, flush=True)
    gen = torch.Generator().manual_seed(R + C)
    s = torch.randn(R, C, generator=gen) * eps ** 0.5
    gamma = (1 + 0.1 * torch.randn(C, generator=gen)).to(BF16)
    dy = torch.randn(R, C, generator=gen).to(BF16)
    ds = torch.empty(R, C, device=DEV)
    sd, gd, dyd = s.to(DEV), gamma.to(DEV), dy.to(DEV)
    pcpp.pcpp_rms_norm_backward(R, C, eps, pcpp.PCPP_DTYPE_F32, sd, gd, dyd, None, ds, None, None, 0)
    torch.cuda.synchronize()
    eps = float(torch.tensor(eps))  # as the call has it
    s, w = s.to(F64), gamma.to(F64) * dy.to(F64)
    want, _ = ref.rms_norm_backward(s, gamma.to(F64), dy.to(F64), None, eps)
    rstd = 1 / torch.sqrt(s.square().mean(-1, keepdim=True) + eps)
    part = rstd * (w.abs() + (s * rstd).abs() * w.square().mean(-1, keepdim=True).sqrt())
    worst = float(((ds.cpu().to(F64) - want).abs() / (2.0 ** -18 * part)).nan_to_num(float("inf")).max())
    print(f"worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0
