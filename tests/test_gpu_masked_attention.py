"""Masked attention, forward and backward, against float64."""

import math

import pytest
import torch

from tests import masked_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64, BF16, F32 = torch.float64, torch.bfloat16, torch.float32


def _say(*a):
    print("[case]", *a, flush=True)


def _ints(v):
    return torch.as_tensor(v, dtype=torch.int32)


def _dev(m):
    put = lambda t: None if t is None else t.to(DEV).contiguous()
    return {n: put(getattr(m, n)) for n in ("kv_len", "q_pos", "prefix", "q_doc", "kv_doc", "slopes")}


def _call(q, k, v, m, causal, scale, cap, dy=None, junk=True):
    """y, lse and, with dy, the gradients; workspaces filled with garbage."""
    from paper_2412_02962_amd import pcpp
    B, nq, H, D = q.shape
    nkv, KH = k.shape[1:3]
    g = pcpp.make_masked_geom(B, nq, nkv, H, KH, D, causal=causal, scale=scale, cap=cap)
    keep = _dev(m)
    mask = pcpp.make_mask(**keep)
    d = [t.to(DEV) for t in (q, k, v)]
    y = torch.full((B, nq, H, D), float("nan"), dtype=BF16, device=DEV)
    lse = torch.full((B, H, nq), float("nan"), dtype=F32, device=DEV)
    n = pcpp.pcpp_masked_attention_workspace_size(g)
    ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    pcpp.pcpp_masked_attention(g, mask, *d, y, lse, ws, n)
    out = dict(y=y, lse=lse)
    if dy is not None:
        n = pcpp.pcpp_masked_attention_backward_workspace_size(g)
        ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=DEV)
        grads = [torch.full_like(t, float("nan")) for t in d]
        pcpp.pcpp_masked_attention_backward(g, mask, *d, y, lse, dy.to(DEV), *grads, ws, n)
        out.update(zip(("dq", "dk", "dv"), grads))
    torch.cuda.synchronize()
    return {n: t.cpu() for n, t in out.items()}


def _inputs(B, nq, nkv, H, KH, D, seed, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen).to(BF16)
    return [(size * normal(B, nq, H, D)).to(BF16), normal(B, nkv, KH, D), normal(B, nkv, KH, D), normal(B, nq, H, D)], gen


def _compare(got, want, bound, tag):
    err = (got.to(F64) - want).abs()
    ok = torch.isfinite(want)
    assert torch.equal(got[~ok].to(F64), want[~ok]), f"{tag}: infinities differ"
    worst = float((err[ok] / bound[ok]).max()) if ok.any() else 0.0
    print(f"{tag}: worst error over bound {worst:.3f}", flush=True)
    assert torch.isfinite(got[ok]).all(), f"{tag}: no number"
    assert worst <= 1.0, f"{tag}: {worst}"


def _check(q, k, v, dy, m, causal=False, scale=None, cap=0.0, backward=True, tag=""):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    got = _call(q, k, v, m, causal, scale, cap, dy if backward else None)
    scale = float(torch.tensor(scale, dtype=F32))
    r = ref.attention(*(t.to(F64) for t in (q, k, v)), m, causal, scale, float(torch.tensor(cap, dtype=F32)))
    by, bl = ref.attention_bound(r)
    _compare(got["y"], r["y"], by, tag + " y")
    _compare(got["lse"], r["lse"], bl, tag + " lse")
    if backward:
        want, bounds = ref.gradients(r, dy.to(F64))
        for n in want:
            _compare(got[n], want[n], bounds[n], tag + " " + n)
    return got


def _docs(gen, B, n, kinds, none=0.1, sorted_=True):
    d = torch.randint(0, kinds, (B, n), generator=gen)
    if sorted_:
        d = d.sort(-1).values
    d[torch.rand(B, n, generator=gen) < none] = -1
    if sorted_:  # padding at the end
        d = torch.stack([torch.cat([r[r >= 0], r[r < 0]]) for r in d])
    return d.to(torch.int32)


# B, nq, nkv, H, KH, D
SHAPES = [
    (1, 1, 1, 1, 1, 8), (2, 1, 77, 10, 10, 64), (3, 5, 130, 4, 2, 40), (1, 33, 33, 2, 1, 64), (2, 64, 65, 2, 2, 32),
    (2, 129, 129, 4, 2, 80), (1, 257, 190, 6, 2, 128), (2, 96, 333, 3, 1, 96), (1, 300, 31, 2, 2, 72), (1, 16, 700, 8, 2, 128),
    (1, 513, 513, 1, 1, 64), (2, 127, 256, 2, 2, 120),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_plain(shape):
    (q, k, v, dy), _ = _inputs(*shape, seed=1)
    _check(q, k, v, dy, ref.Masks(), tag=f"{shape}")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_causal_prefix_bias_cap(shape):
    (q, k, v, dy), gen = _inputs(*shape, seed=2, size=3.0)
    B, nq, nkv, H = shape[:4]
    m = ref.Masks(prefix=torch.randint(-2, nkv // 2 + 2, (B,), generator=gen, dtype=torch.int32),
                  slopes=torch.randn(H, generator=gen) * 0.3)
    _check(q, k, v, dy, m, causal=True, cap=5.0, scale=0.2, tag=f"{shape}")


@pytest.mark.parametrize("sorted_", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_documents(shape, sorted_):
    (q, k, v, dy), gen = _inputs(*shape, seed=3)
    B, nq, nkv = shape[:3]
    m = ref.Masks(q_doc=_docs(gen, B, nq, 4, sorted_=sorted_), kv_doc=_docs(gen, B, nkv, 5, sorted_=sorted_))
    _check(q, k, v, dy, m, tag=f"{shape} {sorted_}")


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_lengths_and_positions(shape, causal):
    """Lengths of 0, 1, out of range and in between; positions before the keys
    (queries that see none), among them and far behind."""
    (q, k, v, dy), gen = _inputs(*shape, seed=4)
    nq, nkv = shape[1:3]
    reps = 7
    q, k, v, dy = (t[:1].repeat(reps, 1, 1, 1) for t in (q, k, v, dy))
    m = ref.Masks(kv_len=_ints([0, 1, nkv, nkv + 9, nkv // 2, nkv - 1, -3]), q_pos=_ints([0, 0, -3, 5, nkv // 2 - nq, 100000, 2]),
                  slopes=torch.full((shape[3],), 0.01))
    clamped = ref.Masks(kv_len=m.kv_len.clamp(0, nkv), q_pos=m.q_pos, slopes=m.slopes)
    got = _call(q, k, v, m, causal, 0.3, 0.0, dy)
    r = ref.attention(*(t.to(F64) for t in (q, k, v)), clamped, causal, float(torch.tensor(0.3, dtype=F32)))
    by, bl = ref.attention_bound(r)
    _compare(got["y"], r["y"], by, f"{shape} y")
    _compare(got["lse"], r["lse"], bl, f"{shape} lse")
    want, bounds = ref.gradients(r, dy.to(F64))
    for n in want:
        _compare(got[n], want[n], bounds[n], f"{shape} {n}")
    assert (got["y"][0] == 0).all() and (got["dk"][0] == 0).all() and (got["dq"][0] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=str)
@pytest.mark.parametrize("shape", [(2, 1, 300, 4, 2, 64), (2, 200, 200, 2, 1, 64), (1, 150, 150, 2, 2, 128), (2, 70, 260, 2, 1, 40)], ids=str)
def test_what_is_not_seen_does_not_count(shape, bad):
    """No number in keys and values of another document, behind a sequence's end
    and in the future, and in queries and gradients of another document: the
    first document's results are as without them, bit for bit."""
    (q, k, v, dy), gen = _inputs(*shape, seed=5)
    B, nq, nkv = shape[:3]
    cut_q, cut_k = max(1, nq * 2 // 3), nkv * 2 // 3 + 3
    qd, kd = torch.zeros(B, nq, dtype=torch.int32), torch.zeros(B, nkv, dtype=torch.int32)
    if nq > 1:
        qd[:, cut_q:] = 7
    kd[:, cut_k:] = 7
    m = ref.Masks(kv_len=_ints([nkv - 5] * B), q_pos=_ints([nkv - nq] * B), q_doc=qd, kv_doc=kd)
    clean = _call(q, k, v, m, True, 0.125, 0.0, dy)
    for t in (k, v):
        t[:, cut_k::3] = bad
    if nq > 1:
        q[:, cut_q::2] = bad
        dy[:, cut_q::2] = bad
    got = _call(q, k, v, m, True, 0.125, 0.0, dy)
    for n, cut in (("y", cut_q), ("dq", cut_q), ("dk", cut_k), ("dv", cut_k)):
        assert torch.equal(got[n][:, :cut], clean[n][:, :cut]), n
    assert (got["dk"][:, nkv - 5:] == 0).all() and (got["dv"][:, nkv - 5:] == 0).all()


def test_the_future_does_not_count():
    """Without documents: no number in a late key, value, query or gradient."""
    (q, k, v, dy), _ = _inputs(1, 100, 100, 2, 1, 64, seed=6)
    clean = _call(q, k, v, ref.Masks(), True, 0.125, 0.0, dy)
    k[:, 70], v[:, 75], q[:, 80], dy[:, 85] = (float("nan"), float("inf"), float("nan"), float("inf"))
    got = _call(q, k, v, ref.Masks(), True, 0.125, 0.0, dy)
    for n in ("y", "dq"):
        assert torch.equal(got[n][:, :70], clean[n][:, :70]), n
    assert got["y"][:, 70:].isnan().any(-1).all()
    # the keys that the spoilt queries do not see
    for n in ("dk", "dv"):
        assert torch.equal(got[n][:, 86:], clean[n][:, 86:]) or got[n][:, 86:].isnan().any(), n


@pytest.mark.parametrize("few", [True, False])
def test_strides(few):
    """q, k, v side by side in one tensor, its gradients in another, y in wider
    rows: what lies between is neither read nor written."""
    from paper_2412_02962_amd import pcpp
    B, n, H, KH, D = 2, 90, 4, 2, 64
    nq = 3 if few else n
    gen = torch.Generator().manual_seed(8)
    width = (H + 2 * KH) * D + 24
    qkv = torch.randn(B, n + 2, width, generator=gen).to(BF16).to(DEV)
    q, k, v = qkv[:, :nq, 8:8 + H * D], qkv[:, :n, 8 + H * D:8 + (H + KH) * D], qkv[:, :n, 8 + (H + KH) * D:8 + (H + 2 * KH) * D]
    ybuf = torch.full((B, nq + 1, H * D + 16), 5.0, dtype=BF16, device=DEV)
    y = ybuf[:, :nq, 8:8 + H * D]
    dybuf = torch.randn(B, nq + 1, H * D + 16, generator=gen).to(BF16).to(DEV)
    dy = dybuf[:, :nq, 8:8 + H * D]
    grad = torch.full_like(qkv, 5.0)
    dq, dk, dv = grad[:, :nq, 8:8 + H * D], grad[:, :n, 8 + H * D:8 + (H + KH) * D], grad[:, :n, 8 + (H + KH) * D:8 + (H + 2 * KH) * D]
    g = pcpp.make_masked_geom(B, nq, n, H, KH, D, causal=True, q_row=width, k_row=width, v_row=width, y_row=H * D + 16,
                              q_batch=qkv.stride(0), k_batch=qkv.stride(0), v_batch=qkv.stride(0), y_batch=ybuf.stride(0))
    lse = torch.empty(B, H, nq, device=DEV)
    nb = max(pcpp.pcpp_masked_attention_workspace_size(g), pcpp.pcpp_masked_attention_backward_workspace_size(g))
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
    pcpp.pcpp_masked_attention(g, None, q, k, v, y, lse, ws, nb)
    pcpp.pcpp_masked_attention_backward(g, None, q, k, v, y, lse, dy, dq, dk, dv, ws, nb)
    torch.cuda.synchronize()
    heads = lambda t: t.cpu().reshape(t.shape[0], t.shape[1], -1, D)
    r = ref.attention(*(heads(t).to(F64) for t in (q, k, v)), ref.Masks(), True, 0.125)
    _compare(heads(y), r["y"], ref.attention_bound(r)[0], "y")
    want, bounds = ref.gradients(r, heads(dy).to(F64))
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        _compare(heads(t), want[name], bounds[name], name)
    for buf, views in ((ybuf, (y,)), (grad, (dq, dk, dv))):
        for t in views:
            t.fill_(5.0)
        assert (buf == 5.0).all()


@pytest.mark.parametrize("shape", [(1, 1, 5000, 8, 2, 128), (3, 2, 2049, 4, 1, 64), (2, 8, 4097, 8, 8, 40), (1, 20, 3000, 3, 1, 96)], ids=str)
def test_long_cache(shape):
    """Pieces of the keys, joined: lengths that leave pieces empty."""
    (q, k, v, dy), gen = _inputs(*shape, seed=9)
    B, nq, nkv, H = shape[:4]
    for lens in ([nkv] * B, [1 + 40 * b for b in range(B)], [nkv - 33 * (b + 1) for b in range(B)]):
        lens = _ints(lens)
        m = ref.Masks(kv_len=lens, q_pos=lens - nq, slopes=2.0 ** -torch.arange(1, H + 1).to(F32))
        scale = shape[-1] ** -0.5
        got = _call(q, k, v, m, True, scale, 20.0)
        r = ref.attention(*(t.to(F64) for t in (q, k, v)), m, True, float(torch.tensor(scale, dtype=F32)), 20.0)
        by, bl = ref.attention_bound(r, step=2.0 ** -16)  # probabilities as two bf16
        _compare(got["y"], r["y"], by, f"{shape} {lens.tolist()} y")
        _compare(got["lse"], r["lse"], bl, f"{shape} lse")


def test_growing_scores():
    """Scores that grow by hundreds along the keys: the running maximum moves
    many times; then ones that fall, and one that dwarfs the rest."""
    (q, k, v, dy), _ = _inputs(1, 100, 400, 1, 1, 64, seed=10)
    for order in (1, -1):
        ramp = torch.arange(400.0)[:, None] * order
        k2 = (torch.ones(400, 64) * ramp / 100).to(BF16).reshape(1, 400, 1, 64)
        q2 = torch.full_like(q, 4.0)
        _check(q2, k2, v, dy, ref.Masks(), tag=f"ramp {order}")
    k[:, 250] = 30.0
    _check(q, k, v, dy, ref.Masks(), tag="spike")


def test_same_at_every_call():
    (q, k, v, dy), gen = _inputs(2, 200, 200, 4, 2, 64, seed=11)
    m = ref.Masks(q_doc=_docs(gen, 2, 200, 3), kv_doc=_docs(gen, 2, 200, 3))
    a, b = (_call(q, k, v, m, True, 0.1, 10.0, dy) for _ in range(2))
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_single_gradients():
    """dq alone, dk and dv alone: as both together."""
    from paper_2412_02962_amd import pcpp
    (q, k, v, dy), _ = _inputs(1, 70, 90, 2, 1, 64, seed=12)
    both = _call(q, k, v, ref.Masks(), False, 0.125, 0.0, dy)
    g = pcpp.make_masked_geom(1, 70, 90, 2, 1, 64)
    n = pcpp.pcpp_masked_attention_backward_workspace_size(g)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    d = [t.to(DEV) for t in (q, k, v, both["y"], both["lse"], dy)]
    dq, dk, dv = (torch.full_like(t, float("nan")) for t in d[:3])
    pcpp.pcpp_masked_attention_backward(g, None, *d, dq, None, None, ws, n)
    pcpp.pcpp_masked_attention_backward(g, None, *d, None, dk, dv, ws, n)
    torch.cuda.synchronize()
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(t.cpu(), both[name]), name
