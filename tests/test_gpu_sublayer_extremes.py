"""Signalling NaN, products that pass float32's range on the way to a value
within it, and infinite weights in the feed-forward sub-layer's operators."""

import pytest
import torch

from tests import ff_reference as ref

pytestmark = pytest.mark.gpu
DEV, F64, BF16, U8 = "cuda", torch.float64, torch.bfloat16, torch.uint8


def _say(*a):
    print("[case]", *a, flush=True)


def _worst(err, bound):
    worst = float((err / bound).nan_to_num(float("inf")).max())
    print(f"worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0


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


# rows and channels of one wavefront a row, of four, and of four for few rows
NORM_SHAPES = [(3, 64), (300, 1280), (9, 640), (2, 4096)]


def _small_rows(R, C, eps):
    gen = torch.Generator().manual_seed(R + C)
    s = torch.randn(R, C, generator=gen) * eps ** 0.5
    s[R // 2] = 0
    return gen, s, float(torch.tensor(eps))  # eps as the call has it


@pytest.mark.parametrize("R,C", NORM_SHAPES)
def test_the_norm_with_a_large_gamma(R, C):
    """rstd about 2^49 and gamma about 2^100: s rstd gamma is finite, and zero
    where s is; rstd gamma is not a float32.  y is its own rounding and that of
    a few float32 operations, whose errors are relative: 2^-18."""
    from paper_2412_02962_amd import pcpp
    _say("large gamma", R, C)
    gen, s, eps = _small_rows(R, C, 1e-30)
    gamma = (2.0 ** 100 * (1 + 0.1 * torch.randn(C, generator=gen))).to(BF16)
    y = torch.empty(R, C, device=DEV, dtype=BF16)
    sd, gd = s.to(DEV), gamma.to(DEV)
    pcpp.pcpp_rms_norm(R, C, eps, pcpp.PCPP_DTYPE_F32, sd, None, gd, None, y)
    torch.cuda.synchronize()
    want = ref.rms_norm(s.to(F64), gamma.to(F64), eps)
    _worst((y.cpu().to(F64) - want).abs(), (ref.HALF_BF16 + 2.0 ** -18) * want.abs() + 1e-30)


@pytest.mark.parametrize("R,C", NORM_SHAPES)
def test_the_norms_gradient_with_a_large_dy(R, C):
    """rstd about 2^49, dy about 2^100 and gamma about 2^-70: dy n and dy gamma
    rstd are finite, dy rstd is not.  What cancels carries 2^-18 of its size, as
    do dgamma's terms, whose float32 sum adds them in any order."""
    from paper_2412_02962_amd import pcpp
    _say("large dy", R, C)
    gen, s, eps = _small_rows(R, C, 1e-30)
    gamma = (2.0 ** -70 * (1 + 0.1 * torch.randn(C, generator=gen))).to(BF16)
    dy = (2.0 ** 100 * torch.randn(R, C, generator=gen)).to(BF16)
    ds, dgamma = torch.empty(R, C, device=DEV), torch.empty(C, device=DEV, dtype=BF16)
    n = pcpp.pcpp_rms_norm_backward_workspace_size(R, C)
    ws = torch.empty(n, dtype=U8, device=DEV)
    sd, gd, dyd = s.to(DEV), gamma.to(DEV), dy.to(DEV)
    pcpp.pcpp_rms_norm_backward(R, C, eps, pcpp.PCPP_DTYPE_F32, sd, gd, dyd, None, ds, dgamma, ws, n)
    torch.cuda.synchronize()
    s, dy, gamma = s.to(F64), dy.to(F64), gamma.to(F64)
    want, want_g = ref.rms_norm_backward(s, gamma, dy, None, eps)
    rstd = 1 / torch.sqrt(s.square().mean(-1, keepdim=True) + eps)
    w = (dy * gamma).abs()
    part = rstd * (w + (s * rstd).abs() * w.square().mean(-1, keepdim=True).sqrt())
    _worst((ds.cpu().to(F64) - want).abs(), 2.0 ** -24 * want.abs() + 2.0 ** -18 * part)
    terms = (dy * s * rstd).abs().sum(0)
    _worst((dgamma.cpu().to(F64) - want_g).abs(), ref.HALF_BF16 * want_g.abs() + 2.0 ** -18 * terms)


@pytest.mark.parametrize("M", [1, 3, 8, 9, 16, 17, 130])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_an_infinite_weight(M, kind):
    """An infinity in ff2_w makes its column of y infinite with h's sign, however
    many tokens a call has; the other columns stay as they are without it."""
    from paper_2412_02962_amd import pcpp
    _say("infinite weight", M, kind)
    C, F = 64, 128
    gen = torch.Generator().manual_seed(M)
    x = torch.randn(M, C, generator=gen).to(BF16)
    w = dict(ff1_w=(torch.randn(2 * F, C, generator=gen) * C ** -0.5).to(BF16), ff1_b=torch.zeros(2 * F, dtype=BF16),
             ff2_w=torch.randn(C, F, generator=gen).to(BF16), ff2_b=torch.zeros(C, dtype=BF16))
    # a whole h, and one that bf16 holds exactly (its second half is zero)
    w["ff1_w"][40], w["ff1_w"][F + 40] = 0, 0
    w["ff1_b"][40], w["ff1_b"][F + 40] = 1.0, 100.0
    outs = []
    g = pcpp.make_ff_geom(M, C, F, pcpp.PCPP_ACT_SILU if kind == "silu" else pcpp.PCPP_ACT_GELU)
    n = pcpp.pcpp_gated_ff_workspace_size(g)
    ws = torch.empty(n, dtype=U8, device=DEV)
    for infinite in (False, True):
        if infinite:
            w["ff2_w"][5, 17], w["ff2_w"][30, 40] = float("inf"), -float("inf")
        wd, y = {k: v.to(DEV) for k, v in w.items()}, torch.empty(M, C, device=DEV, dtype=BF16)
        pcpp.pcpp_gated_ff(g, pcpp.make_ff_weights(wd), x.to(DEV), y, None, None, ws, n)
        torch.cuda.synchronize()
        outs.append(y.cpu())
    h = ref.gated_ff(x.to(F64), {k: v.to(F64) for k, v in w.items()}, kind)[1]
    assert bool((h[:, 17].abs() > 1e-6).all()) and bool((h[:, 40] == 100).all())
    keep = [c for c in range(C) if c not in (5, 30)]
    assert torch.equal(outs[0][:, keep], outs[1][:, keep])
    assert torch.equal(outs[1][:, 5].to(F64), torch.sign(h[:, 17]) * float("inf"))
    assert bool((outs[1][:, 30] == -float("inf")).all())
