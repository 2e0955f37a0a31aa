"""Infinities that are seen: the masked attention's results by the formula, the
same in tiles that all queries see whole and in ones that some see a part of."""

import pytest
import torch

from tests import masked_reference as ref
from tests.test_gpu_masked_attention import BF16, F32, F64, _call, _compare, _inputs

pytestmark = pytest.mark.gpu

INF = float("inf")
HUGE = 1e100  # in float64 as good as infinite: its tanh is 1, its exponential 0 or beyond every sum
N = 400       # four blocks of 128: the spoilt tokens' tiles are whole for some and cut for others
# B, H, KH, D
SHAPES = [(1, 2, 1, 64), (14, 2, 2, 128), (20, 2, 1, 40), (2, 6, 2, 96)]


def _finite(t, as_):
    t = t.to(F64)
    return torch.where(t.isinf(), t.sign() * as_, t)


def _masks(kind, B):
    if kind == "causal":
        return ref.Masks(), True
    doc = torch.zeros(B, N, dtype=torch.int32)
    doc[:, 150:] = 1
    doc[:, 290:] = -1
    return ref.Masks(q_doc=doc, kv_doc=doc), False


def _expected(q, k, v, dy, m, causal, scale, cap):
    """Results and bounds of inputs whose infinities saturate their scores, and
    where dq and dk are no number: 0 times an infinity that is seen."""
    d64 = [t.to(F64) for t in (v, dy)]
    r = ref.attention(_finite(q, HUGE), _finite(k, HUGE), d64[0], m, causal, scale, cap)
    r0 = ref.attention(_finite(q, 0.0), _finite(k, 0.0), d64[0], m, causal, scale, cap)
    # a saturated score has no error but its transform's, 3 cap; the operands of
    # the products over keys and queries are 0 there, as their weights are
    for n in ("E", "qh", "kh"):
        r[n] = r0[n]
    want, bounds = ref.gradients(r, d64[1])
    by, bl = ref.attention_bound(r)
    want.update(y=r["y"], lse=r["lse"])
    bounds.update(y=by, lse=bl)
    B, _, H, D = q.shape
    KH = k.shape[2]
    ok = ref.seen(m, B, N, N, causal, "cpu").to(F64)[:, None]
    heads = lambda t: t.isinf().to(F64).permute(0, 2, 1, 3)
    nan = dict(dq=(ok @ heads(k).repeat_interleave(H // KH, 1) > 0).permute(0, 2, 1, 3),
               dk=(ok.transpose(2, 3) @ heads(q) > 0).reshape(B, KH, H // KH, N, D).any(2).permute(0, 2, 1, 3))
    return want, bounds, nan


def _check(q, k, v, dy, kind, cap, tag):
    m, causal = _masks(kind, q.shape[0])
    scale = float(torch.tensor(q.shape[-1] ** -0.5, dtype=F32))
    got = _call(q, k, v, m, causal, scale, cap, dy)
    want, bounds, nan = _expected(q, k, v, dy, m, causal, scale, cap)
    for n in want:
        t, w = got[n], want[n]
        if n in nan:
            assert torch.equal(t.isnan(), nan[n]), f"{tag} {n}: {int((t.isnan() != nan[n]).sum())} are, or are not, numbers"
            t, w = t.clone(), w.clone()
            t[nan[n]] = 0
            w[nan[n]] = 0
        _compare(t, w, bounds[n], f"{tag} {n}")


@pytest.mark.parametrize("kind", ["causal", "documents"])
@pytest.mark.parametrize("bad", [INF, -INF], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_keys_under_a_cap(shape, bad, kind):
    """Scores of plus and minus the cap: y and lse are finite, and so are dq's
    other channels, dk and dv."""
    B, H, KH, D = shape
    (q, k, v, dy), _ = _inputs(B, N, N, H, KH, D, seed=81)
    k[:, 10, 0, 3] = bad
    k[:, 130, -1, D - 1] = bad
    k[:, 201, 0, 0] = -bad
    _check(q, k, v, dy, kind, 5.0, f"{shape} {bad} {kind}")


@pytest.mark.parametrize("kind", ["causal", "documents"])
@pytest.mark.parametrize("bad", [INF, -INF], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_queries_under_a_cap(shape, bad, kind):
    B, H, KH, D = shape
    (q, k, v, dy), _ = _inputs(B, N, N, H, KH, D, seed=82)
    q[:, 40, 0, 5] = bad
    q[:, 200, -1, D - 2] = bad
    q[:, 270, 0, 1] = -bad
    _check(q, k, v, dy, kind, 5.0, f"{shape} {bad} {kind}")


@pytest.mark.parametrize("kind", ["causal", "documents"])
@pytest.mark.parametrize("bad", [INF, -INF], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_keys_that_nobody_takes(shape, bad, kind):
    """No cap, scores of -infinity: weights of 0."""
    B, H, KH, D = shape
    (q, k, v, dy), _ = _inputs(B, N, N, H, KH, D, seed=83)
    q[..., 2] = (-q[..., 2].float().abs() - 0.1).to(BF16) if bad > 0 else (q[..., 2].float().abs() + 0.1).to(BF16)
    k[:, 11, :, 2] = bad
    k[:, 131, 0, 2] = bad
    k[:, 202, -1, 2] = bad
    _check(q, k, v, dy, kind, 0.0, f"{shape} {bad} {kind}")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scores_of_plus_infinity_are_no_numbers(shape):
    """No cap, an infinite key or query: nothing of a query that sees it is a
    number, and everything before it is as without it."""
    B, H, KH, D = shape
    (q, k, v, dy), _ = _inputs(B, N, N, H, KH, D, seed=84)
    q[..., 2] = (q[..., 2].float().abs() + 0.1).to(BF16)
    scale = D ** -0.5
    clean = _call(q, k, v, ref.Masks(), True, scale, 0.0, dy)
    spoilt = k.clone()
    spoilt[:, 130, :, 2] = INF
    got = _call(q, spoilt, v, ref.Masks(), True, scale, 0.0, dy)
    for n in ("y", "dq"):
        assert torch.equal(got[n][:, :130], clean[n][:, :130]) and got[n][:, 130:].isnan().all(), n
    assert got["dk"].isnan().all() and got["dv"].isnan().all()
    spoilt = q.clone()
    spoilt[:, 200, :, 2] = INF
    got = _call(spoilt, k, v, ref.Masks(), True, scale, 0.0, dy)
    others = torch.arange(N) != 200
    for n in ("y", "dq"):
        assert torch.equal(got[n][:, others], clean[n][:, others]) and got[n][:, 200].isnan().all(), n
    for n in ("dk", "dv"):
        assert got[n][:, :201].isnan().all() and torch.equal(got[n][:, 201:], clean[n][:, 201:]), n


@pytest.mark.parametrize("bad", [float("nan"), INF, -INF], ids=str)
@pytest.mark.parametrize("shape", [(1, 100, 2, 1, 64), (40, 100, 4, 2, 64), (20, 200, 4, 4, 128), (30, 150, 2, 1, 40)], ids=str)
def test_queries_and_gradients_of_the_past_do_not_count(shape, bad):
    """Causal, without documents: no number in an early query and an early
    gradient; keys behind them do not see it, bit for bit."""
    B, n, H, KH, D = shape
    (q, k, v, dy), _ = _inputs(B, n, n, H, KH, D, seed=85)
    clean = _call(q, k, v, ref.Masks(), True, 0.125, 0.0, dy)
    q[:, 30], dy[:, 20] = bad, bad
    got = _call(q, k, v, ref.Masks(), True, 0.125, 0.0, dy)
    for t in ("dk", "dv"):
        assert torch.isfinite(clean[t]).all() and torch.equal(got[t][:, 31:], clean[t][:, 31:]), t
        assert got[t][:, :21].isnan().all() or t == "dv" and not torch.isfinite(got[t][:, :21]).any(), t
    others = torch.ones(n, dtype=torch.bool)
    others[30] = False
    assert torch.equal(got["y"][:, others], clean["y"][:, others])
    others[20] = False
    assert torch.equal(got["dq"][:, others], clean["dq"][:, others])
