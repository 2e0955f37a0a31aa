"""GroupNorm with its activation over the most tokens that an image may have,
2^30: the same 2^17 rows again and again, whose statistics are theirs."""

import pytest
import torch

from tests import norm_act_reference as ref
from tests.test_gpu_norm_act import BF16, DEV, F64, _inputs, _near

pytestmark = pytest.mark.gpu


def test_the_most_tokens():
    from paper_2412_02962_amd import pcpp
    R, N, C, G, eps = 1 << 13, 1 << 17, 8, 2, 1e-5
    x, gamma, beta, dy = _inputs(1, N, C, BF16, seed=71)
    d = [t.to(F64) for t in (x, gamma, beta, dy)]
    r = ref.forward(*d[:3], G, eps, "silu", 0.0, 0, 0, BF16)
    (dx, dgamma, dbeta), (bx, bg, bb) = ref.backward(r, d[1], d[3], "silu", 0.0, 0, 0, BF16)
    # Besides: a thread merges 2^30 / 512 / 256 / 8 = 1024 runs of rows, each off
    # by 2^-24 of the mean or the sum, and 512 chunks are merged: 2^-13 of the
    # mean of the magnitudes, in n, in both means and in the columns' sums.
    da = 1.2  # |SiLU'|
    w = d[3].abs() * da * d[1].abs()
    e_n = 2.0 ** -13 * (r["n"].abs() + r["rstd"].max() * d[0].abs().mean())
    by = r["bound"] + da * d[1].abs() * e_n
    bx = bx + r["rstd"].max() * (2.0 ** -13 * (w + w.mean() + r["n"].abs() * (w * r["n"].abs()).mean()) + w * e_n + (w.mean() + w) * e_n)
    sums = (d[3].abs() * da * (1 + r["n"].abs())).sum((0, 1))

    g = pcpp.make_norm_act_geom(1, R * N, C, G, eps=eps)
    n = pcpp.pcpp_group_norm_act_workspace_size(g)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    xs, dys = (t.to(DEV)[0].repeat(R, 1) for t in (x, dy))
    y = torch.empty_like(xs)
    stats = torch.empty(1, G, 2, device=DEV)
    params = [t.to(DEV) for t in (gamma, beta)]
    grads = [torch.empty_like(t) for t in params]
    print("[case] forward", flush=True)
    pcpp.pcpp_group_norm_act(g, xs, *params, None, 0, y, stats, ws, n)
    torch.cuda.synchronize()
    print("[case] backward", flush=True)
    pcpp.pcpp_group_norm_act_backward(g, xs, *params, stats, None, 0, dys, dys, *grads, ws, n)  # dx in dy's place
    torch.cuda.synchronize()
    for name, t, want, bound in (("y", y, r["y"], by), ("dx", dys, dx, bx)):
        t = t.reshape(R, N, C)
        for i in range(0, R, 512):
            assert torch.equal(t[i:i + 512], t[:1].expand(512, N, C)), (name, i)
        _near(t[:1].cpu(), want, bound, name)
    for name, t, want, bound in (("dgamma", grads[0], dgamma, bg), ("dbeta", grads[1], dbeta, bb)):
        _near(t.cpu(), R * want, R * (bound + 2.0 ** -13 * sums), name)
