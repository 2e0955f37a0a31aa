"""GroupNorm with its activation and dropout, forward and backward, against
float64."""

import pytest
import torch

from tests import norm_act_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64, BF16, F32 = torch.float64, torch.bfloat16, torch.float32
SEED, FIRST, DRAW = 0xABCDEF123, 40, 2


def _state():
    return torch.tensor([SEED, FIRST], dtype=torch.int64, device=DEV)


def _call(x, gamma, beta, G, eps, kind, p, dy, in_place=False, params=True):
    from paper_2412_02962_amd import pcpp
    B, N, C = x.shape
    act = dict(none=pcpp.PCPP_ACT_NONE, silu=pcpp.PCPP_ACT_SILU, gelu=pcpp.PCPP_ACT_GELU)[kind]
    dtype = pcpp.PCPP_DTYPE_F32 if x.dtype == F32 else pcpp.PCPP_DTYPE_BF16
    g = pcpp.make_norm_act_geom(B, N, C, G, act, dtype, eps, p)
    n = pcpp.pcpp_group_norm_act_workspace_size(g)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    x, gamma, beta, dy = (t.to(DEV) for t in (x, gamma, beta, dy))
    y = torch.full_like(x, float("nan"))
    stats = torch.full((B, G, 2), float("nan"), device=DEV)
    st = _state() if p else None
    pcpp.pcpp_group_norm_act(g, x, gamma, beta, st, DRAW, y, stats, ws, n)
    ws.fill_(0xFF)
    dx = dy if in_place else torch.full_like(x, float("nan"))
    dgamma, dbeta = (torch.full_like(gamma, float("nan")) if params else None for _ in range(2))
    pcpp.pcpp_group_norm_act_backward(g, x, gamma, beta, stats, st, DRAW, dy, dx, dgamma, dbeta, ws, n)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu() for t in (y, stats, dx, dgamma, dbeta)]


def _near(got, want, bound, tag):
    err = (got.to(F64) - want).abs()
    worst = float((err / bound).max())
    print(f"{tag}: worst error over bound {worst:.3f}", flush=True)
    assert torch.isfinite(got).all() and worst <= 1.0, f"{tag}: {worst}"


def _inputs(B, N, C, dtype, seed, mean=1.0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)
    x = (n(B, N, C) * (0.3 + torch.rand(C, generator=gen)) + mean * n(C)).to(dtype)
    return x, (1 + 0.2 * n(C)).to(BF16), (0.2 * n(C)).to(BF16), n(B, N, C).to(dtype)


# B, N, C, G
SHAPES = [(1, 1, 8, 1), (1, 1, 8, 8), (2, 7, 40, 5), (1, 133, 64, 64), (2, 300, 320, 32), (3, 77, 960, 32), (1, 64, 2560, 32),
          (1, 50, 2552, 8), (2, 31, 2560, 1), (1, 2100, 128, 16), (2, 1000, 640, 32), (1, 9000, 72, 24), (1, 19, 1280, 256)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=str)
@pytest.mark.parametrize("kind,p", [("silu", 0.1), ("gelu", 0.0), ("none", 0.5), ("gelu", 0.25), ("silu", 0.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_float64(shape, kind, p, dtype):
    B, N, C, G = shape
    x, gamma, beta, dy = _inputs(B, N, C, dtype, seed=N + C)
    eps = 1e-5
    y, stats, dx, dgamma, dbeta = _call(x, gamma, beta, G, eps, kind, p, dy)
    d = [t.to(F64) for t in (x, gamma, beta, dy)]
    r = ref.forward(*d[:3], G, eps, kind, p, SEED, FIRST + DRAW, dtype)
    _near(stats[..., 0], r["mean"], r["mean_bound"] + 1e-30, "mean")
    _near(stats[..., 1], r["rstd"], r["rstd_bound"], "rstd")
    _near(y, r["y"], r["bound"], "y")
    want, bounds = ref.backward(r, d[1], d[3], kind, p, SEED, FIRST + DRAW, dtype)
    for got, w, b, tag in zip((dx, dgamma, dbeta), want, bounds, ("dx", "dgamma", "dbeta")):
        _near(got, w, b, tag)


def test_far_from_zero():
    """A mean of a thousand deviations: no difference of large sums."""
    x, gamma, beta, dy = _inputs(1, 500, 64, F32, seed=1, mean=0.0)
    x = x + 1000
    y, stats, dx, _, _ = _call(x, gamma, beta, 4, 1e-5, "none", 0.0, dy)
    d = [t.to(F64) for t in (x, gamma, beta, dy)]
    r = ref.forward(*d[:3], 4, 1e-5, "none", 0.0, 0, 0, F32)
    # rstd of deviations, each off by half a step of the mean's size
    assert ((stats[..., 1].to(F64) / r["rstd"] - 1).abs() <= 2.0 ** -10).all()
    _near(y, r["y"], r["bound"] + 2.0 ** -10 * r["n"].abs() * d[1].abs(), "y")


def test_constant_group():
    x = torch.full((1, 10, 16), 3.0)
    _, gamma, beta, dy = _inputs(1, 10, 16, F32, seed=2)
    y, stats, dx, dgamma, dbeta = _call(x, gamma, beta, 2, 1e-5, "none", 0.0, dy)
    assert torch.equal(y, beta.float().expand(1, 10, 16)) and (stats[..., 0] == 3).all() and (dgamma == 0).all()


def test_dropped_gradients_are_not_read_as_numbers():
    x, gamma, beta, dy = _inputs(1, 64, 64, F32, seed=3)
    keep = ref.kept(64 * 64, 0.5, SEED, FIRST + DRAW).reshape(1, 64, 64)
    a = _call(x, gamma, beta, 8, 1e-5, "silu", 0.5, torch.where(keep, dy, 0.0))
    b = _call(x, gamma, beta, 8, 1e-5, "silu", 0.5, torch.where(keep, dy, float("nan")))
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_in_place_and_without_parameters():
    x, gamma, beta, dy = _inputs(2, 100, 320, BF16, seed=4)
    a = _call(x, gamma, beta, 32, 1e-5, "silu", 0.1, dy)
    b = _call(x, gamma, beta, 32, 1e-5, "silu", 0.1, dy, in_place=True, params=False)
    assert torch.equal(a[2], b[2]) and b[3] is None


def test_agrees_with_the_inference_form():
    """pcpp_group_norm with SiLU on the same input: both within a step."""
    from paper_2412_02962_amd import pcpp
    x, gamma, beta, dy = _inputs(2, 1024, 640, BF16, seed=5)
    y = _call(x, gamma, beta, 32, 1e-5, "silu", 0.0, dy)[0]
    n = pcpp.pcpp_group_norm_workspace_size(2, 1024, 640, 32)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    other = torch.empty(2, 1024, 640, dtype=BF16, device=DEV)
    pcpp.pcpp_group_norm(2, 1024, 640, 32, 1e-5, 1, x.to(DEV), gamma.to(DEV), beta.to(DEV), other, ws, n)
    other = other.cpu().to(F64)
    assert ((y.to(F64) - other).abs() <= 2 * 2.0 ** -8 * other.abs() + 3e-6).all()
