"""Arrays past 2^32 elements through the feed-forward sub-layer's operators: the
same rows over and over, so that every repeat has to come out like the first
and the first can be compared with the reference."""

import pytest
import torch

from tests import ff_reference as ref
from tests.test_gpu_feed_forward import Call, _check, _dev, _f64, _inputs

pytestmark = pytest.mark.gpu
DEV, F64, BF16, U8 = "cuda", torch.float64, torch.bfloat16, torch.uint8


def _repeats_alike(t, rows, tag):
    for i in range(rows, t.shape[0], rows):
        assert torch.equal(t[i:i + rows], t[:rows]), (tag, i)


def test_many_tokens():
    rows, repeats, C, F, kind = 4099, 130, 64, 8192, "gelu"
    M = rows * repeats
    print("[case] many tokens", M, C, F, flush=True)
    x, w, dy = _inputs(rows, C, F, 5)
    c = Call(M, C, F, kind, _dev(w))
    assert c.codes.numel() > 2 ** 32
    xd, dyd = x.to(DEV).repeat(repeats, 1), dy.to(DEV).repeat(repeats, 1)
    c.forward(xd)
    torch.cuda.synchronize()
    x64, w64, dy64 = x.to(DEV, F64), _f64(c.wd), dy.to(DEV, F64)
    _check(c.y[:rows], ref.gated_ff(x64, w64, kind)[2].cpu(), ref.gated_ff_bound(x64, w64, kind).cpu(), "y")
    for t, tag in ((c.y, "y"), (c.codes, "codes"), (c.scales, "scales")):
        _repeats_alike(t, rows, tag)
    c.backward(xd, dyd)
    torch.cuda.synchronize()
    kept = ref.from_8bit(c.codes[:rows].cpu(), c.scales[:rows].cpu()).to(DEV)
    want = ref.gated_ff_backward(x64, w64, kept, dy64, kind)
    bound = ref.gated_ff_backward_bound(x64, w64, kept, dy64, kind)
    _check(c.dx[:rows], want["dx"].cpu(), bound["dx"].cpu(), "dx")
    _repeats_alike(c.dx, rows, "dx")
    for k, t in c.grads.items():  # every repeat adds the same, errors too; float32 sums of M / 16 parts
        size = want[k].abs() + bound[k]
        _check(t, repeats * want[k].cpu(), (repeats * (bound[k] + M / 16 * 2.0 ** -24 * size)).cpu(), k)


def test_many_rows():
    from paper_2412_02962_amd import pcpp
    rows, repeats, C = 1009, 530, 8192
    R, code = rows * repeats, pcpp.PCPP_DTYPE_BF16
    print("[case] many rows", R, C, flush=True)
    gen = torch.Generator().manual_seed(3)
    x, a = (torch.randn(rows, C, generator=gen).to(DEV, BF16) for _ in range(2))
    gamma = (1 + 0.1 * torch.randn(C, generator=gen)).to(DEV, BF16)
    xd, ad = x.repeat(repeats, 1), a.repeat(repeats, 1)
    assert xd.numel() > 2 ** 32
    y, codes = torch.empty_like(xd), torch.empty((R, C), dtype=U8, device=DEV)
    scales = torch.empty((R, C // 32), dtype=U8, device=DEV)
    pcpp.pcpp_rms_norm(R, C, 1e-6, code, xd, ad, gamma, xd, y, codes, scales)
    torch.cuda.synchronize()
    s = x.to(F64) + a.to(F64)
    want = ref.rms_norm(s, gamma.to(F64), 1e-6)
    _check(y[:rows], want.cpu(), (ref.HALF_BF16 * want.abs() + 2.0 ** -12).cpu(), "y")
    for t, tag in ((xd, "sum"), (y, "y"), (codes, "codes"), (scales, "scales")):
        _repeats_alike(t, rows, tag)
    ad.fill_(0)
    pcpp.pcpp_checkpoint_load(R, C, code, codes, scales, ad)
    torch.cuda.synchronize()
    assert torch.equal(ad[:rows].cpu().to(F64), ref.from_8bit(codes[:rows].cpu(), scales[:rows].cpu()))
    _repeats_alike(ad, rows, "load")
    codes2, scales2 = torch.zeros_like(codes), torch.zeros_like(scales)
    pcpp.pcpp_checkpoint_save(R, C, code, ad, codes2, scales2)
    torch.cuda.synchronize()
    # of values that are codes already: the same ones, by a scale that is perhaps smaller
    back = torch.empty_like(ad)
    pcpp.pcpp_checkpoint_load(R, C, code, codes2, scales2, back)
    torch.cuda.synchronize()
    _repeats_alike(back, rows, "save")
    assert torch.equal(back[:rows], ad[:rows])
    # ds of the same rows; dgamma is left out (its sum has a test of its own)
    pcpp.pcpp_rms_norm_backward(R, C, 1e-6, code, xd, gamma, y, None, back, None, None, 0)
    torch.cuda.synchronize()
    _repeats_alike(back, rows, "ds")
    s16 = xd[:rows].to(F64)
    want, _ = ref.rms_norm_backward(s16, gamma.to(F64), y[:rows].to(F64), None, 1e-6)
    rstd = 1 / torch.sqrt(s16.square().mean(-1, keepdim=True) + 1e-6)
    g = (y[:rows].to(F64) * gamma.to(F64)).abs()
    part = rstd * (g + (s16 * rstd).abs() * g.square().mean(-1, keepdim=True).sqrt())
    # where s and so dy are zero, ds, its error and its bound are: 0 / 0 without the last term
    _check(back[:rows], want.cpu(), (ref.HALF_BF16 * want.abs() + 2.0 ** -18 * part + 1e-30).cpu(), "ds")
