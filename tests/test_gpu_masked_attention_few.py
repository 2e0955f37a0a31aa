"""Masked attention where few workgroups of 32 queries share the keys: the
probabilities are two bf16 there, 2^-16 of their value, and y and lse are held to
that."""

import pytest
import torch

from tests import masked_reference as ref
from tests.test_gpu_masked_attention import DEV, F32, F64, _call, _compare, _dev, _docs, _inputs, _ints

pytestmark = pytest.mark.gpu

# B, nq, nkv, H, KH, D
SHAPES = [(1, 1, 1, 1, 1, 8), (2, 1, 77, 10, 10, 64), (3, 5, 130, 4, 2, 40), (1, 33, 33, 2, 1, 64), (2, 64, 65, 2, 2, 32), (2, 129, 129, 4, 2, 80),
          (1, 257, 190, 6, 2, 128), (2, 96, 333, 3, 1, 96), (1, 16, 700, 8, 2, 128), (1, 513, 513, 1, 1, 64), (2, 127, 256, 2, 2, 120),
          (4, 1000, 1000, 1, 1, 128), (1, 434, 4000, 4, 1, 96)]


def _step(B, nq, nkv, H, KH, D):
    """Of the probabilities: this form works up to 64 queries of the heads that
    share keys, or at most 128 times 32 of them in all on 128 keys or more.  (One
    of the shapes, 66 queries on 33 keys, is not.)"""
    rows = H // KH * nq
    return 2.0 ** -16 if rows <= 64 or (B * KH * -(-rows // 32) <= 128 and nkv >= 128) else ref.HALF


@pytest.mark.parametrize("kind", ["plain", "causal", "documents"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_probabilities_of_two_bf16(shape, kind):
    (q, k, v, _), gen = _inputs(*shape, seed=91, size=2.0)
    B, nq, nkv, H = shape[:4]
    m, causal, cap = ref.Masks(), False, 0.0
    if kind == "causal":
        m, causal, cap = ref.Masks(slopes=torch.randn(H, generator=gen) * 0.1, prefix=_ints([nkv // 3] * B)), True, 8.0
    elif kind == "documents":
        m = ref.Masks(q_doc=_docs(gen, B, nq, 4), kv_doc=_docs(gen, B, nkv, 4), kv_len=_ints([max(1, nkv - 9 * b) for b in range(B)]))
    scale = float(torch.tensor(0.15, dtype=F32))
    got = _call(q, k, v, m, causal, scale, cap)
    r = ref.attention(*(t.to(DEV).to(F64) for t in (q, k, v)), ref.Masks(**_dev(m)), causal, scale, cap)
    by, bl = ref.attention_bound(r, step=_step(*shape))
    _compare(got["y"], r["y"].cpu(), by.cpu(), f"{shape} {kind} y")
    _compare(got["lse"], r["lse"].cpu(), bl.cpu(), f"{shape} {kind} lse")
