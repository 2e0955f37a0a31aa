"""GPU parity of pcpp_rms_norm, pcpp_rms_norm_backward and the 8-bit
checkpoints with the float64 reference.

y and ds (bf16) are one rounding, 2^-8 of their magnitude at most, of a
float32 computation whose own error (a sum of at most 8192 squares in a tree,
a square root and a division) is far below 2^-12 of the row's rms; ds in
float32 is held to 2^-18 of the row's rms.  A code is off by half a step at
most (2^-4 of the value, 2^-10 of the scale below the smallest normal code),
and by that of y's float32 error in addition."""

import math

import pytest
import torch

from tests import ff_reference as ref

pytestmark = pytest.mark.gpu

DEV, EPS = "cuda:0", 1e-6
F32, F64, BF16, U8 = torch.float32, torch.float64, torch.bfloat16, torch.uint8

SHAPES = [(1, 8), (1, 64), (3, 32), (2, 1280), (77, 640), (300, 2048), (257, 1288), (5, 2080), (33, 4096), (2, 8192),
          (1025, 96), (4099, 320)]


def _say(*a):
    print("[case]", *a, flush=True)


def _types(stream):
    from paper_2412_02962_amd import pcpp
    return (F32, pcpp.PCPP_DTYPE_F32) if stream == "f32" else (BF16, pcpp.PCPP_DTYPE_BF16)


def _stream_rows(gen, R, C, dtype):
    x = torch.randn((R, C), generator=gen) * torch.exp(torch.randn((R, 1), generator=gen))
    return (x * (1 + 9 * (torch.rand((1, C), generator=gen) > 0.95))).to(dtype)


def _check(err, bound, tag):
    worst = float((err / bound).max())
    print(f"{tag}: worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0, (tag, worst)


@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", SHAPES)
def test_rms_norm(R, C, stream):
    from paper_2412_02962_amd import pcpp
    _say("rms norm", R, C, stream)
    dtype, code = _types(stream)
    gen = torch.Generator().manual_seed(R * 10007 + C)
    x, r = _stream_rows(gen, R, C, dtype), torch.randn((R, C), generator=gen).to(BF16)
    gamma = (1 + 0.3 * torch.randn(C, generator=gen)).to(BF16)
    xd, rd, gd = x.to(DEV), r.to(DEV), gamma.to(DEV)
    eight = C % 32 == 0
    for addend in (r, None):
        s32 = x.to(F32) + (addend.to(F32) if addend is not None else 0)
        want = ref.rms_norm(s32.to(F64), gamma.to(F64), EPS)
        bound = ref.HALF_BF16 * want.abs() + 2.0 ** -12 * want.square().mean(-1, keepdim=True).sqrt()
        guard = torch.full((R + 2, C), 7.0, dtype=BF16, device=DEV)      # the rows around stay
        y, sum_out = guard[1:-1], torch.empty_like(xd)
        codes = torch.full((R, C), 7, dtype=U8, device=DEV) if eight else None
        scales = torch.full((R, C // 32), 7, dtype=U8, device=DEV) if eight else None
        pcpp.pcpp_rms_norm(R, C, EPS, code, xd, None if addend is None else rd, gd, sum_out, y, codes, scales)
        torch.cuda.synchronize()
        assert torch.equal(sum_out.cpu(), s32.to(dtype))
        _check((y.cpu().to(F64) - want).abs(), bound, f"y {R} x {C}")
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
        if eight:
            val = ref.from_8bit(codes.cpu(), scales.cpu())
            e = torch.exp2(ref.scale_exponents(want).to(F64)).repeat_interleave(32, 1)
            rms = want.square().mean(-1, keepdim=True).sqrt()
            half = torch.maximum(ref.HALF_E4M3 * want.abs(), 2.0 ** -10 * e)
            _check((val - want).abs(), half * (1 + 2.0 ** -10) + 2.0 ** -18 * rms, "8-bit y")
        # only one of the outputs, in place
        x2 = xd.clone()
        y2 = torch.empty_like(y)
        pcpp.pcpp_rms_norm(R, C, EPS, code, x2, None if addend is None else rd, gd, x2, y2)
        torch.cuda.synchronize()
        assert torch.equal(x2, sum_out) and torch.equal(y2, y)


@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", SHAPES)
def test_rms_norm_backward(R, C, stream):
    from paper_2412_02962_amd import pcpp
    _say("rms norm backward", R, C, stream)
    dtype, code = _types(stream)
    gen = torch.Generator().manual_seed(R * 10009 + C)
    s, dy = _stream_rows(gen, R, C, dtype), torch.randn((R, C), generator=gen).to(BF16)
    d0 = torch.randn((R, C), generator=gen).to(dtype)
    gamma = (1 + 0.3 * torch.randn(C, generator=gen)).to(BF16)
    sd, dyd, d0d, gd = (t.to(DEV) for t in (s, dy, d0, gamma))
    wsb = pcpp.pcpp_rms_norm_backward_workspace_size(R, C)
    ws = torch.full((wsb,), 0xA5, dtype=U8, device=DEV)
    for ds_in in (d0, None):
        want, want_g = ref.rms_norm_backward(s.to(F64), gamma.to(F64), dy.to(F64),
                                             None if ds_in is None else ds_in.to(F64), EPS)
        ds, dgamma = torch.empty_like(sd), torch.empty_like(gd)
        pcpp.pcpp_rms_norm_backward(R, C, EPS, code, sd, gd, dyd, None if ds_in is None else d0d, ds, dgamma, ws, wsb)
        torch.cuda.synchronize()
        # what cancels: rstd w, rstd n mean(w n) and ds_in, each with a few float32 roundings
        rstd = 1 / torch.sqrt(s.to(F64).square().mean(-1, keepdim=True) + EPS)
        w = (dy.to(F64) * gamma.to(F64)).abs()
        part = rstd * (w + (s.to(F64) * rstd).abs() * w.square().mean(-1, keepdim=True).sqrt())
        if ds_in is not None:
            part = part + ds_in.to(F64).abs()
        _check((ds.cpu().to(F64) - want).abs(), (ref.HALF_BF16 if stream == "bf16" else 2.0 ** -24) * want.abs() +
               2.0 ** -18 * part, f"ds {R} x {C}")
        n = (dy.to(F64) * s.to(F64) * rstd)
        _check((dgamma.cpu().to(F64) - want_g).abs(), ref.HALF_BF16 * want_g.abs() + 2.0 ** -18 * n.square().sum(0).sqrt() +
               1e-12, "dgamma")
        d2 = d0d.clone() if ds_in is not None else None
        if d2 is not None:   # in place, and without dgamma
            pcpp.pcpp_rms_norm_backward(R, C, EPS, code, sd, gd, dyd, d2, d2, None)
            torch.cuda.synchronize()
            assert torch.equal(d2, ds)


def test_rms_norm_rows_do_not_touch_each_other():
    """A row of NaN, of infinities, of zeros: only that row is affected."""
    from paper_2412_02962_amd import pcpp
    _say("rms norm special rows")
    R, C = 9, 640
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((R, C), generator=gen)
    gamma = torch.ones(C, dtype=BF16)
    bad = x.clone()
    bad[2], bad[4, 17], bad[6] = float("nan"), float("inf"), 0.0
    out = []
    for t in (x, bad):
        y = torch.empty((R, C), dtype=BF16, device=DEV)
        codes, scales = torch.empty((R, C), dtype=U8, device=DEV), torch.empty((R, C // 32), dtype=U8, device=DEV)
        pcpp.pcpp_rms_norm(R, C, EPS, pcpp.PCPP_DTYPE_F32, t.to(DEV), None, gamma.to(DEV), None, y, codes, scales)
        torch.cuda.synchronize()
        out.append((y.cpu(), ref.from_8bit(codes.cpu(), scales.cpu())))
    keep = [r for r in range(R) if r not in (2, 4, 6)]
    assert torch.equal(out[0][0][keep], out[1][0][keep]) and torch.equal(out[0][1][keep], out[1][1][keep])
    y, v = out[1]
    assert y[2].isnan().all() and v[2].isnan().all() and y[4, 17].isnan() and v[4, 17].isnan()
    assert (y[4, :17] == 0).all() and (y[6] == 0).all() and (v[6] == 0).all()


CHECK_SHAPES = [(1, 32), (3, 96), (7, 640), (129, 2560), (1000, 64), (11, 65536)]


@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", CHECK_SHAPES)
def test_checkpoint_codes_are_exact(R, C, stream):
    """No arithmetic but the rounding: codes, scales and values read back are
    the reference's, over 60 octaves, with zeros, subnormal codes, ties,
    infinities and NaN among them."""
    from paper_2412_02962_amd import pcpp
    _say("checkpoint", R, C, stream)
    dtype, code = _types(stream)
    gen = torch.Generator().manual_seed(R + C)
    x = torch.randn((R, C), generator=gen) * torch.exp2(torch.randint(-40, 20, (R, C // 32, 1), generator=gen).float()
                                                        ).expand(R, C // 32, 32).reshape(R, C)
    x = torch.where(torch.rand((R, C), generator=gen) < 0.1, torch.round(x * 8) / 8, x)     # ties
    flat = x.reshape(-1)
    for i, v in enumerate((float("inf"), float("nan"), -float("inf"), 0.0, -0.0, 1e-45, 3e38, -448.0, 448.5)):
        flat[(i * 37 + 5) % flat.numel()] = v
    x = x.to(dtype)
    codes, scales = torch.empty((R, C), dtype=U8, device=DEV), torch.empty((R, C // 32), dtype=U8, device=DEV)
    pcpp.pcpp_checkpoint_save(R, C, code, x.to(DEV), codes, scales)
    torch.cuda.synchronize()
    want_c, want_s = ref.to_8bit(x)
    got = codes.cpu()
    nan = (want_c & 127) == 127
    assert torch.equal(scales.cpu(), want_s)
    assert ((got & 127) == 127)[nan].all() and torch.equal(got[~nan], want_c[~nan])
    for out, name in ((F32, pcpp.PCPP_DTYPE_F32), (BF16, pcpp.PCPP_DTYPE_BF16)):
        back = torch.empty((R, C), dtype=out, device=DEV)
        pcpp.pcpp_checkpoint_load(R, C, name, codes, scales, back)
        torch.cuda.synchronize()
        want = ref.from_8bit(want_c, want_s).to(out)
        assert torch.equal(torch.nan_to_num(back.cpu(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
