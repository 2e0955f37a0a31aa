"""The masked attention's logarithms of the sums of exp(s), which the backward
pass takes its probabilities from: held to float32's roundings, whichever form
works a call."""

import pytest
import torch

from tests import masked_reference as ref
from tests.test_gpu_masked_attention import BF16, DEV, F32, F64, _call, _compare, _dev, _inputs, _ints

pytestmark = pytest.mark.gpu


def _bound(r, nkv):
    """The scores' (2 E), the logarithm's and its result's, and the sum's own: of
    a lane's keys, 32 of every 64, one after the other in a step and the steps
    one after the other, and a few to join lanes, wavefronts and pieces."""
    lse = r["lse"].abs().nan_to_num(posinf=0)
    return 2 * r["E"][..., 0] + 2.0 ** -21 * lse + (nkv / 64 + 64) * 2.0 ** -24


def _dominated(shape, seed):
    """Scores of which one, behind the first 64 keys, is 1 to 12 above the
    others, by query."""
    (q, k, v, dy), gen = _inputs(*shape, seed=seed)
    B, nq, nkv, H, KH, D = shape
    q, k = 0.1 * q.float(), 0.1 * k.float()
    q[..., 0] = torch.linspace(1, 12, nq)[None, :, None]
    k[..., 0] = 0
    k[:, nkv // 2 + 3, :, 0] = D ** 0.5  # (the scale's inverse)
    return (q.to(BF16), k.to(BF16), v, dy), gen


# B, nq, nkv, H, KH, D: blocks of 128 queries to a workgroup; few workgroups of
# many queries; few queries, in pieces of the keys too
SHAPES = [(17, 129, 700, 4, 2, 64), (9, 257, 1390, 6, 2, 128), (20, 96, 4000, 6, 2, 96), (40, 70, 327, 2, 2, 40),
          (1, 300, 4000, 2, 2, 64), (2, 1, 333, 8, 2, 128), (1, 5, 9000, 4, 1, 64)]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_key_dominates(shape, masked):
    (q, k, v, _), gen = _dominated(shape, seed=61)
    B, nq, nkv, H, KH, D = shape
    m = ref.Masks()
    if masked:
        doc = torch.zeros(B, nkv, dtype=torch.int32)
        doc[:, ::7] = 1
        m = ref.Masks(kv_len=_ints([nkv - 3 * b for b in range(B)]), q_pos=_ints([nkv - nq] * B), kv_doc=doc,
                      q_doc=torch.zeros(B, nq, dtype=torch.int32))
    scale = float(torch.tensor(D ** -0.5, dtype=F32))
    got = _call(q, k, v, m, masked, scale, 0.0)
    r = ref.attention(*(t.to(DEV).to(F64) for t in (q, k, v)), ref.Masks(**_dev(m)), masked, scale)
    _compare(got["lse"], r["lse"].cpu(), _bound(r, nkv).cpu(), f"{shape} {masked} lse")
    by, _ = ref.attention_bound(r)
    _compare(got["y"], r["y"].cpu(), by.cpu(), f"{shape} {masked} y")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_capped_and_biased(shape):
    (q, k, v, _), gen = _inputs(*shape, seed=62, size=3.0)
    H, nkv = shape[3], shape[2]
    m = ref.Masks(slopes=torch.rand(H, generator=gen) * 0.02)
    got = _call(q, k, v, m, True, 0.2, 10.0)
    r = ref.attention(*(t.to(DEV).to(F64) for t in (q, k, v)), ref.Masks(**_dev(m)), True, float(torch.tensor(0.2, dtype=F32)), 10.0)
    _compare(got["lse"], r["lse"].cpu(), _bound(r, nkv).cpu(), f"{shape} lse")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_y_does_not_depend_on_lse(shape):
    """With lse and without: the same bits."""
    from paper_2412_02962_amd import pcpp
    (q, k, v, _), _ = _dominated(shape, seed=63)
    B, nq, nkv, H, KH, D = shape
    g = pcpp.make_masked_geom(*shape)
    n = pcpp.pcpp_masked_attention_workspace_size(g)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    d = [t.to(DEV) for t in (q, k, v)]
    y = torch.full((B, nq, H, D), float("nan"), dtype=BF16, device=DEV)
    pcpp.pcpp_masked_attention(g, None, *d, y, None, ws, n)
    torch.cuda.synchronize()
    assert torch.equal(y.cpu(), _call(q, k, v, ref.Masks(), False, D ** -0.5, 0.0)["y"])
