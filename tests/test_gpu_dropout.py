"""Dropout with the residual's addition: masks bit for bit, values in float32."""

import pytest
import torch

from tests import norm_act_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64, BF16, F32 = torch.float64, torch.bfloat16, torch.float32


def _run(x, residual, y, p, state, draw):
    from paper_2412_02962_amd import pcpp
    code = {F32: pcpp.PCPP_DTYPE_F32, BF16: pcpp.PCPP_DTYPE_BF16}
    pcpp.pcpp_dropout(x.numel(), code[x.dtype], code[y.dtype], p, state, draw, x, residual, y)
    torch.cuda.synchronize()
    return y


def _state(seed, first):
    wrap = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v
    return torch.tensor([wrap(seed), wrap(first)], dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2560, 8191, 8192, 100003])
@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)], ids=str)
def test_values_and_mask(n, types):
    gen = torch.Generator().manual_seed(n)
    x, res = torch.randn(n, generator=gen).to(types[0]), torch.randn(n, generator=gen).to(types[1])
    for p, seed, first, draw in ((0.1, 5, 0, 0), (0.5, 2 ** 64 - 3, 2 ** 64 - 2, 7), (0.0, 1, 1, 1), (1.0, 1, 1, 1), (0.9, 2 ** 40, 3, 2 ** 64 - 1)):
        for r in (None, res):
            y = torch.full((n + 16,), float("nan"), dtype=types[1], device=DEV)
            _run(x.to(DEV), None if r is None else r.to(DEV), y[:n], p, _state(seed, first), draw)
            got = y.cpu()
            assert got[n:].isnan().all()
            d = ref.dropped(x.to(F64), p, seed, first + draw)
            want = d + (0 if r is None else r.to(F64))
            # the product and the sum in float32, the result once
            bound = ref.HALF[types[1]] * want.abs() + 2.0 ** -23 * (d.abs() + want.abs()) + 1e-38
            assert ((got[:n].to(F64) - want).abs() <= bound).all(), (p, r is None)
            if r is None:
                gone = ~ref.kept(n, p, seed, first + draw) if p > 0 else torch.zeros(n, dtype=torch.bool)
                assert (got[:n][gone] == 0).all()


def test_no_number_is_dropped():
    n, p = 4096, 0.5
    keep = ref.kept(n, p, 9, 4)
    for bad in (float("nan"), float("inf")):
        x = torch.where(keep, 1.0, bad).to(BF16).to(DEV)
        y = _run(x, None, torch.empty(n, dtype=BF16, device=DEV), p, _state(9, 4), 0)
        assert torch.equal(y.cpu() != 0, keep) and torch.isfinite(y).all()


def test_in_place():
    n, p = 5003, 0.25
    gen = torch.Generator().manual_seed(3)
    x, res = torch.randn(n, generator=gen).to(DEV), torch.randn(n, generator=gen).to(DEV)
    st = _state(1, 2)
    want = _run(x, res, torch.empty_like(x), p, st, 3)
    for over in ("x", "residual"):
        a, b = x.clone(), res.clone()
        assert torch.equal(_run(a, b, a if over == "x" else b, p, st, 3), want)


def test_gradient_is_the_same_mask():
    n, p = 10007, 0.3
    gen = torch.Generator().manual_seed(4)
    x, dy = torch.randn(n, generator=gen).to(DEV), torch.randn(n, generator=gen).to(DEV)
    st = _state(77, 5)
    y = _run(x, None, torch.empty_like(x), p, st, 11)
    dx = _run(dy, None, torch.empty_like(dy), p, st, 11)
    f = ref.factor(p)
    assert torch.equal(dx != 0, y != 0)
    d = torch.randn(n, generator=gen).to(DEV)
    up, dn = (_run(x + s * d, None, torch.empty_like(x), p, st, 11) for s in (0.5, -0.5))
    got, want = float(((up - dn).double() * dy.double()).sum()), float((dx.double() * d.double()).sum())
    assert abs(got - want) <= 2.0 ** -20 * f * float((dy.abs().double() * (x.abs() + d.abs()).double()).sum())


def test_beyond_2_to_32_elements():
    """The last elements of an array of 2^32 + 19: their place takes 64 bits."""
    n, p = 2 ** 32 + 19, 0.4
    x = torch.ones(n, dtype=BF16, device=DEV)
    y = _run(x, None, x, p, _state(3, 1), 0)
    first = n - 19 - 8 * 1000
    assert torch.equal(y[first:].cpu() != 0, ref.kept(n - first, p, 3, 1, first=first))
    assert torch.equal(y[:8000].cpu() != 0, ref.kept(8000, p, 3, 1))


def test_captured_and_replayed():
    """A graph takes a new mask when the state on the device moves on, the same
    one when it does not; eager work and synchronizations between."""
    n, p = 3001, 0.2
    x = torch.randn(n, device=DEV)
    y, st = torch.empty_like(x), _state(6, 100)
    _run(x, None, y, p, st, 1)
    graph = torch.cuda.CUDAGraph()
    from paper_2412_02962_amd import pcpp
    with torch.cuda.graph(graph):
        pcpp.pcpp_dropout(n, 0, 0, p, st, 1, x, None, y)
        st[1:].add_(10)
    for step in range(4):
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = _run(x, None, torch.empty_like(x), p, _state(6, 100 + 10 * step), 1)
        assert torch.equal(y, want), step
