"""The float64 reference of masked attention: gradients against automatic
differentiation and central differences, values against hand-made cases."""

import math

import pytest
import torch

from tests import masked_reference as ref

F64 = torch.float64


def _case(seed, H=4, KH=2):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, dtype=F64)
    q, k, v, dy = n(2, 5, H, 8), n(2, 7, KH, 8), n(2, 7, KH, 8), n(2, 5, H, 8)
    m = ref.Masks(kv_len=torch.tensor([7, 5]), q_pos=torch.tensor([2, -1]), prefix=torch.tensor([0, 2]),
                  q_doc=torch.tensor([[0, 0, 1, 1, -1], [3, 3, 3, 3, 3]]), kv_doc=torch.tensor([[0, 0, 0, 1, 1, 1, -1], [3, 3, 0, 3, 3, 3, 3]]),
                  slopes=n(H) * 0.2)
    return q, k, v, dy, m


@pytest.mark.parametrize("cap", [0.0, 2.0])
@pytest.mark.parametrize("seed", [0, 1])
def test_gradients_by_differentiation_and_differences(seed, cap):
    q, k, v, dy, m = _case(seed)
    r = ref.attention(q, k, v, m, True, 0.4, cap)
    want, bounds = ref.gradients(r, dy)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    (ref.attention(*leaves, m, True, 0.4, cap)["y"] * dy).sum().backward()
    for leaf, n in zip(leaves, ("dq", "dk", "dv")):
        assert torch.allclose(leaf.grad, want[n], rtol=1e-10, atol=1e-12), n
        assert (bounds[n] > 0).all()
    f = lambda *a: float((ref.attention(*a, m, True, 0.4, cap)["y"] * dy).sum())
    gen = torch.Generator().manual_seed(seed + 50)
    for x, n in ((0, "dq"), (1, "dk"), (2, "dv")):
        d = torch.randn((q, k, v)[x].shape, generator=gen, dtype=F64)
        h = 1e-5
        up, dn = ([t + s * h * d if i == x else t for i, t in enumerate((q, k, v))] for s in (1, -1))
        assert abs((f(*up) - f(*dn)) / (2 * h) - float((want[n] * d).sum())) < 1e-7


def test_library_attention_agrees():
    q, k, v, _, _ = _case(3)
    r = ref.attention(q, k, v, ref.Masks(q_pos=torch.tensor([0, 0])), True)
    rep = lambda t: t.permute(0, 2, 1, 3).repeat_interleave(2, 1)
    want = torch.nn.functional.scaled_dot_product_attention(q.permute(0, 2, 1, 3), rep(k), rep(v), is_causal=True)
    assert torch.allclose(r["yh"], want, atol=1e-12)


def test_masks_by_hand():
    m = ref.Masks(kv_len=torch.tensor([4]), q_pos=torch.tensor([1]), prefix=torch.tensor([1]), q_doc=torch.tensor([[0, 2, -1]]),
                  kv_doc=torch.tensor([[0, 0, 2, 2, 2]]))
    ok = ref.seen(m, 1, 3, 5, True, "cpu")[0]
    assert ok.tolist() == [[True, True, False, False, False], [False, False, True, False, False], [False] * 5]
    q, k = torch.zeros(1, 3, 1, 8, dtype=F64), torch.zeros(1, 5, 1, 8, dtype=F64)
    v = torch.arange(5, dtype=F64)[None, :, None, None].expand(1, 5, 1, 8)
    r = ref.attention(q, k, v, m, True)
    assert r["y"][0, :, 0, 0].tolist() == [0.5, 2.0, 0.0]
    assert r["lse"][0, 0, 2] == -math.inf and abs(float(r["lse"][0, 0, 0]) - math.log(2)) < 1e-12
