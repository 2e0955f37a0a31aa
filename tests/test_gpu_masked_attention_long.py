"""Masked attention over long sequences and wide strides, against float64 on
the device; and as a program calls it: in graphs and on other streams."""

import pytest
import torch

from tests import masked_reference as ref
from tests import test_gpu_masked_attention as short
from tests.test_gpu_masked_attention import BF16, DEV, F32, F64, _call, _compare, _dev, _inputs, _ints

pytestmark = pytest.mark.gpu


def _check(q, k, v, dy, m, causal=False, cap=0.0, scale=0.125, few=False, tag=""):
    """_check of the short ones with its reference on the device."""
    got = _call(q, k, v, m, causal, scale, cap, dy)
    md = ref.Masks(**_dev(m))
    r = ref.attention(*(t.to(DEV).to(F64) for t in (q, k, v)), md, causal, scale, cap)
    by, bl = ref.attention_bound(r, step=2.0 ** -16) if few else ref.attention_bound(r)
    _compare(got["y"], r["y"].cpu(), by.cpu(), tag + " y")
    _compare(got["lse"], r["lse"].cpu(), bl.cpu(), tag + " lse")
    want, bounds = ref.gradients(r, dy.to(DEV).to(F64))
    for n in want:
        _compare(got[n], want[n].cpu(), bounds[n].cpu(), tag + " " + n)


# The keys' gradients in pieces of the queries (heads / kv_heads * n_q / 64 tiles
# of them, two or more to a piece), the last ones ragged, some empty.
PIECES = [(1, 577, 513, 4, 1, 64), (1, 1100, 300, 2, 1, 128), (2, 700, 130, 6, 2, 96), (1, 1537, 1, 1, 1, 40)]


@pytest.mark.parametrize("kind", ["plain", "causal", "documents"])
@pytest.mark.parametrize("shape", PIECES, ids=str)
def test_pieces_of_the_queries(shape, kind):
    (q, k, v, dy), gen = _inputs(*shape, seed=21)
    B, nq, nkv, H = shape[:4]
    if kind == "plain":
        m = ref.Masks()
    elif kind == "causal":
        m = ref.Masks(slopes=torch.randn(H, generator=gen) * 0.1, q_pos=_ints([nkv // 2 - nq // 2] * B), prefix=_ints([7] * B))
    else:
        draw = lambda n: torch.randint(-1, 4, (B, n), generator=gen).sort(-1).values.to(torch.int32)
        m = ref.Masks(q_doc=draw(nq), kv_doc=draw(nkv))
    _check(q, k, v, dy, m, causal=kind == "causal", cap=8.0 if kind == "causal" else 0.0, tag=f"{shape} {kind}")


# B, nq, nkv, H, KH, D: sequences enough for blocks of 128 queries to a workgroup
MANY = [(17, 129, 129, 4, 2, 80), (9, 257, 190, 6, 2, 128), (20, 96, 333, 6, 2, 96), (40, 70, 127, 2, 2, 64), (5, 513, 513, 2, 2, 64),
        (12, 127, 256, 4, 4, 120)]


@pytest.mark.parametrize("shape", MANY, ids=str)
def test_blocks_of_queries(shape):
    short.test_plain(shape)
    short.test_causal_prefix_bias_cap(shape)
    for sorted_ in (True, False):
        short.test_documents(shape, sorted_)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 700, 513, 20, 20, 64), (1, 700, 300, 20, 20, 128), (1, 400, 140, 40, 20, 96)], ids=str)
def test_blocks_of_queries_lengths_and_positions(shape, causal):
    short.test_lengths_and_positions(shape, causal)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=str)
@pytest.mark.parametrize("shape", [(12, 200, 200, 2, 1, 64), (14, 150, 150, 2, 2, 128), (20, 200, 260, 2, 1, 40), (20, 200, 260, 2, 1, 96)], ids=str)
def test_blocks_of_queries_what_is_not_seen(shape, bad):
    short.test_what_is_not_seen_does_not_count(shape, bad)


@pytest.mark.parametrize("D", [64, 128])
def test_blocks_of_queries_growing_scores(D):
    """Scores that grow by hundreds along the keys, fall, and one that dwarfs the
    rest: 40 sequences of 100 queries."""
    (q, k, v, dy), _ = _inputs(40, 100, 400, 1, 1, D, seed=27)
    for order in (1, -1):
        ramp = torch.arange(400.0)[:, None] * order
        k2 = (torch.ones(400, D) * ramp / 100).to(BF16).reshape(1, 400, 1, D).repeat(40, 1, 1, 1)
        _check(torch.full_like(q, 4.0), k2, v, dy, ref.Masks(), tag=f"ramp {order}")
    k[:, 250] = 30.0
    _check(q, k, v, dy, ref.Masks(), tag="spike")


@pytest.mark.parametrize("docs", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_several_rounds_of_workgroups(causal, docs):
    """560 blocks of queries and 896 of keys: more than twice 32 to each part of
    the chip, which take them in an order of their own."""
    shape = (4, 777, 777, 20, 4, 40)
    (q, k, v, dy), gen = _inputs(*shape, seed=26)
    doc = torch.randint(-1, 5, (4, 777), generator=gen).sort(-1).values.to(torch.int32) if docs else None
    _check(q, k, v, dy, ref.Masks(q_doc=doc, kv_doc=doc), causal=causal, scale=0.16, tag=f"{causal} {docs}")


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_documents_far_apart(bias, causal):
    """More than 64 tiles of 64 tokens: a document at both ends of a sequence,
    short ones between, long ones, and padding inside."""
    n, H = 9001, 2
    (q, k, v, dy), gen = _inputs(1, n, n, H, 1, 32, seed=22)
    at = torch.arange(n)
    doc = 1 + at // 700
    doc[(at < 100) | (at >= n - 90)] = 0
    doc[(at > 3000) & (at < 3300)] = 50 + at[(at > 3000) & (at < 3300)] // 3
    doc[(at > 6000) & (at < 6200)] = -1
    doc = doc.to(torch.int32)[None]
    m = ref.Masks(q_doc=doc, kv_doc=doc, slopes=torch.tensor([0.001, 0.2]) if bias else None)
    _check(q, k, v, dy, m, causal=causal, scale=0.2, tag=f"{bias} {causal}")


@pytest.mark.parametrize("bias", [False, True])
def test_few_queries_documents_far_apart(bias):
    """Two and three queries of different documents over a cache of many windows
    of tiles, no document in most of them."""
    B, nq, nkv, H = 2, 3, 70001, 2
    (q, k, v, dy), gen = _inputs(B, nq, nkv, H, 1, 64, seed=23)
    kd = torch.full((B, nkv), 9)
    for b, (lo, hi, d) in ((0, (5, 40, 1)), (0, (30000, 30002, 1)), (0, (69990, 70001, 2)), (1, (0, 65000, 4)), (1, (65000, 65100, -5))):
        kd[b, lo:hi] = d
    m = ref.Masks(q_doc=_ints([[1, 2, 8], [4, 5, -1]]), kv_doc=kd.to(torch.int32), slopes=torch.tensor([0.0001, -0.00001]) if bias else None,
                  q_pos=_ints([100, 69000]))
    got = _call(q, k, v, m, False, 0.125, 0.0)
    r = ref.attention(*(t.to(F64) for t in (q, k, v)), m, False, 0.125, 0.0)
    by, bl = ref.attention_bound(r, step=2.0 ** -16)
    _compare(got["y"], r["y"], by, "y")
    _compare(got["lse"], r["lse"], bl, "lse")
    assert (got["y"][0, 2] == 0).all() and (got["y"][1, 1:] == 0).all()


@pytest.mark.parametrize("nq", [1, 100])
def test_offsets_beyond_32_bits(nq):
    """Rows of 64 Ki elements: a sequence's keys over 9 GB, gradients too."""
    from paper_2412_02962_amd import pcpp
    n, row, H, D = 70000, 1 << 16, 2, 64
    gen = torch.Generator(DEV).manual_seed(24)
    cache = torch.empty(n, row, dtype=BF16, device=DEV)
    k, v = cache[None, :, 128:128 + D], cache[None, :, 512:512 + D]
    for t in (k, v):
        t.copy_(torch.randn(t.shape, generator=gen, device=DEV))
    q, dy = (torch.randn(1, nq, H * D, generator=gen, device=DEV).to(BF16) for _ in range(2))
    y, lse = torch.empty_like(q), torch.empty(1, H, nq, device=DEV)
    g = pcpp.make_masked_geom(1, nq, n, H, 1, D, causal=True, k_row=row, v_row=row)
    nb = max(pcpp.pcpp_masked_attention_workspace_size(g), pcpp.pcpp_masked_attention_backward_workspace_size(g))
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    pcpp.pcpp_masked_attention(g, None, q, k, v, y, lse, ws, nb)
    heads = lambda t: t.reshape(1, t.shape[1], -1, D)
    r = ref.attention(*(heads(t).to(F64) for t in (q, k, v)), ref.Masks(), True, 0.125)
    _compare(heads(y).cpu(), r["y"].cpu(), ref.attention_bound(r)[0].cpu(), "y")
    if nq == 1:
        return
    grads = torch.empty_like(cache)
    dq, dk, dv = torch.empty_like(q), grads[None, :, 128:128 + D], grads[None, :, 512:512 + D]
    pcpp.pcpp_masked_attention_backward(g, None, q, k, v, y, lse, dy, dq, dk, dv, ws, nb)
    want, bounds = ref.gradients(r, heads(dy).to(F64))
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        _compare(heads(t).cpu(), want[name].cpu(), bounds[name].cpu(), name)


def _program(nq, n, H, KH, D):
    """A training step's calls on buffers of its own, and those buffers."""
    from paper_2412_02962_amd import pcpp
    B = 2
    gen = torch.Generator().manual_seed(25)
    draw = lambda rows: torch.randint(-1, 3, (B, rows), generator=gen).sort(-1).values.to(torch.int32).to(DEV)
    q, dy = (torch.randn(B, nq, H * D, generator=gen).to(BF16).to(DEV) for _ in range(2))
    k, v = (torch.randn(B, n, KH * D, generator=gen).to(BF16).to(DEV) for _ in range(2))
    masks = dict(q_doc=draw(nq), kv_doc=draw(n), slopes=torch.full((H,), 0.02, device=DEV), kv_len=_ints([n, n - 7]).to(DEV),
                 q_pos=_ints([n - nq, n - nq]).to(DEV))
    g = pcpp.make_masked_geom(B, nq, n, H, KH, D, causal=True, cap=20.0)
    nb = max(pcpp.pcpp_masked_attention_workspace_size(g), pcpp.pcpp_masked_attention_backward_workspace_size(g))
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(t) for t in (q, q, k, v)] + [torch.empty(B, H, nq, device=DEV)]
    m = pcpp.make_mask(**masks)

    def run(o=out, workspace=ws):
        y, dq, dk, dv, lse = o
        pcpp.pcpp_masked_attention(g, m, q, k, v, y, lse, workspace, nb)
        pcpp.pcpp_masked_attention_backward(g, m, q, k, v, y, lse, dy, dq, dk, dv, workspace, nb)
    return run, (q, k, v, dy, masks), out


@pytest.mark.parametrize("shape", [(200, 300, 4, 2, 64), (2, 5000, 8, 2, 128), (700, 513, 4, 1, 96)], ids=str)
def test_captured_and_replayed(shape):
    """Every replay, with other inputs, lengths and positions, is the eager
    result; the program works on the same buffers between the replays."""
    run, (q, k, v, dy, masks), out = _program(*shape)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for step in range(4):
        with torch.no_grad():
            for t in (q, k, v, dy):
                t.copy_(torch.randn_like(t))
            masks["kv_len"].sub_(3 * step)
            masks["q_pos"].sub_(step)
        eager = [torch.empty_like(t) for t in out]
        run(eager)
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b), step


def test_on_another_stream():
    run, _, out = _program(300, 300, 2, 1, 64)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    # two calls at once, each with a workspace of its own
    there = [torch.full_like(t, float("nan")) for t in out]
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(there, ws)
    run()
    torch.cuda.synchronize()
    for a, b, c in zip(want, out, there):
        assert torch.equal(a, b) and torch.equal(a, c)
