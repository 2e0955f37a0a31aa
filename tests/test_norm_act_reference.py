"""The float64 references of dropout and of GroupNorm with its activation:
known vectors, automatic differentiation and central differences."""

import math

import pytest
import torch

from tests import norm_act_reference as ref

F64 = torch.float64


def test_philox_known_answers():
    """The published test vectors of the generator (counter, key -> block)."""
    assert ref.philox(0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 2 ** 64 - 1
    assert ref.philox(ones, ones, ones) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_kept_is_the_generators():
    seed, stream = 0x123456789ABCDEF0, 2 ** 63 + 5
    keep = ref.kept(37, 0.3, seed, stream, first=2 ** 36)
    for i in range(37):
        w = ref.philox((2 ** 36 + i) // 8, stream, seed)[i % 8 // 2]
        assert bool(keep[i]) == ((w >> 16 * (i % 2) & 0xFFFF) >= round(65536 * 0.3))


def test_share_that_is_kept():
    for p in (0.1, 0.5, 0.9):
        n = 1 << 18
        share = float(ref.kept(n, p, 42, 7).double().mean())
        assert abs(share - (1 - p)) < 6 * math.sqrt(p * (1 - p) / n) + 2.0 ** -17


@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients(kind, p):
    gen = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(s, generator=gen, dtype=F64)
    x, gamma, beta, dy = n(2, 5, 12) + 1, n(12), n(12), n(2, 5, 12)
    args = (3, 1e-5, kind, p, 99, 3, torch.float32)
    r = ref.forward(x, gamma, beta, *args)
    (dx, dgamma, dbeta), bounds = ref.backward(r, gamma, dy, kind, p, 99, 3, torch.float32)
    assert all((b > 0).all() for b in bounds)
    leaves = [t.clone().requires_grad_() for t in (x, gamma, beta)]
    (ref.forward(*leaves, *args)["y"] * dy).sum().backward()
    for leaf, want in zip(leaves, (dx, dgamma, dbeta)):
        assert torch.allclose(leaf.grad, want, rtol=1e-9, atol=1e-11)
    f = lambda a: float((ref.forward(a, gamma, beta, *args)["y"] * dy).sum())
    d = n(2, 5, 12)
    assert abs((f(x + 1e-5 * d) - f(x - 1e-5 * d)) / 2e-5 - float((dx * d).sum())) < 1e-7
    if p == 0 and kind == "silu":
        want = torch.nn.functional.silu(torch.nn.functional.group_norm(x.transpose(1, 2), 3, gamma, beta, 1e-5)).transpose(1, 2)
        assert torch.allclose(r["y"], want, atol=1e-10)
