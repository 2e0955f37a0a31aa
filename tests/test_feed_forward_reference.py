"""The float64 reference of the feed-forward sub-layer against independent
forms: central differences for the gradients, torch's e4m3 for the codes."""

import pytest
import torch

from tests import ff_reference as ref

F64 = torch.float64


def _difference(f, x, u, h=1e-5):
    return (f(x + h * u) - f(x - h * u)) / (2 * h)


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_gated_ff_gradients_against_differences(kind):
    gen = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=gen, dtype=F64)
    M, C, F = 5, 32, 64
    x, dy = rnd(M, C), rnd(M, C)
    w = dict(ff1_w=rnd(2 * F, C) * 0.3, ff1_b=rnd(2 * F), ff2_w=rnd(C, F) * 0.2, ff2_b=rnd(C))
    got = ref.gated_ff_backward(x, w, ref.gated_ff(x, w, kind)[0], dy, kind)
    loss = lambda x, w: (ref.gated_ff(x, w, kind)[2] * dy).sum()
    u = rnd(M, C)
    assert torch.allclose((got["dx"] * u).sum(), _difference(lambda t: loss(t, w), x, u), rtol=1e-7)
    for k in w:
        u = rnd(*w[k].shape)
        assert torch.allclose((got[k] * u).sum(), _difference(lambda t: loss(x, {**w, k: t}), w[k], u), rtol=1e-7), k


def test_rms_norm_gradients_against_differences():
    gen = torch.Generator().manual_seed(8)
    rnd = lambda *s: torch.randn(s, generator=gen, dtype=F64)
    s, gamma, dy, ds_in = rnd(4, 24), rnd(24), rnd(4, 24), rnd(4, 24)
    ds, dgamma = ref.rms_norm_backward(s, gamma, dy, ds_in, 1e-3)
    loss = lambda s, g: (ref.rms_norm(s, g, 1e-3) * dy).sum() + (s * ds_in).sum()
    u = rnd(4, 24)
    assert torch.allclose((ds * u).sum(), _difference(lambda t: loss(t, gamma), s, u), rtol=1e-7)
    u = rnd(24)
    assert torch.allclose((dgamma * u).sum(), _difference(lambda t: loss(s, t), gamma, u), rtol=1e-7)


def test_codes_against_torch_e4m3():
    gen = torch.Generator().manual_seed(9)
    v = torch.randn((64, 256), generator=gen) * torch.exp2(torch.randint(-30, 30, (64, 256), generator=gen).float())
    codes, scales = ref.to_8bit(v)
    t = torch.ldexp(v.reshape(64, 8, 32), 127 - scales.to(torch.int32)[..., None])
    assert torch.equal(codes.reshape(64, 8, 32), t.to(torch.float8_e4m3fn).view(torch.uint8))
    want = t.to(torch.float8_e4m3fn).to(F64) * torch.exp2(scales.to(F64) - 127)[..., None]
    assert torch.equal(ref.from_8bit(codes, scales), want.reshape(64, 256))


def test_scales_are_the_smallest_that_hold_the_group():
    v = torch.zeros(6, 32)
    v[0, 3], v[1, 0], v[2, 5], v[3, 1] = 448.0, 448.0 * (1 + 2 ** -23), -1.75 * 2 ** -40, 2.0 ** -126
    v[4, 7], v[4, 8] = float("inf"), 3.0
    _, scales = ref.to_8bit(v)
    assert (scales.to(torch.int32)[:, 0] - 127).tolist() == [0, 1, -48, -117, -7, -117]
