"""Refusals and workspaces of the masked attention's entry points: every call
here fails validation before anything would be enqueued."""

import ctypes

import pytest

A = 1 << 24          # an aligned address; never dereferenced
STEP = 1 << 40       # far enough apart for any size used here
TENSORS = ("q", "k", "v", "y", "lse", "dy", "dq", "dk", "dv")
MASKS = ("kv_len", "q_pos", "prefix", "q_doc", "kv_doc", "slopes")


def _p(name, off=0):
    return A + (TENSORS + MASKS + ("ws",)).index(name) * STEP + off


GEOM = dict(batch=2, n_q=5, n_kv=9, heads=4, kv_heads=2, head_dim=16)
Q_BYTES, K_BYTES = 2 * 5 * 4 * 16 * 2, 2 * 9 * 2 * 16 * 2


def _status(backward, geom=None, mask=None, null_geom=False, null_mask=False, wsb=1 << 30, **over):
    from paper_2412_02962_amd import pcpp
    g = pcpp.make_masked_geom(**{**GEOM, **(geom or {})})
    m = pcpp.pcpp_mask_t(*[(mask or {}).get(n) for n in MASKS])
    a = {n: _p(n) for n in TENSORS + ("ws",)}
    a.update(over)
    gp = None if null_geom else ctypes.byref(g)
    mp = None if null_mask else ctypes.byref(m)
    if backward:
        return pcpp.lib().pcpp_masked_attention_backward(gp, mp, *[a[n] for n in TENSORS], a["ws"], wsb, None)
    return pcpp.lib().pcpp_masked_attention(gp, mp, *[a[n] for n in TENSORS[:5]], a["ws"], wsb, None)


BAD_GEOM = [
    ("EINVAL", dict(batch=0)), ("EINVAL", dict(batch=65536)), ("EINVAL", dict(n_q=0)), ("EINVAL", dict(n_kv=0)),
    ("EINVAL", dict(n_q=(1 << 24) + 1)), ("EINVAL", dict(n_kv=(1 << 24) + 1)), ("EINVAL", dict(heads=0)),
    ("EINVAL", dict(heads=1025, kv_heads=1025)), ("EINVAL", dict(kv_heads=0)), ("EINVAL", dict(kv_heads=3)),
    ("EINVAL", dict(kv_heads=8)), ("EINVAL", dict(causal=2)), ("EINVAL", dict(reserved=1)),
    ("EINVAL", dict(scale=float("nan"))), ("EINVAL", dict(scale=float("inf"))), ("EINVAL", dict(cap=-1.0)),
    ("EINVAL", dict(cap=float("nan"))), ("EINVAL", dict(cap=float("inf"))), ("EINVAL", dict(cap=1e-30, scale=1e30)),
    ("EINVAL", dict(cap=4097.0)),
    ("ENOTSUP", dict(head_dim=4)), ("ENOTSUP", dict(head_dim=12)), ("ENOTSUP", dict(head_dim=136)),
    # launches of 2^32 threads
    ("EINVAL", dict(batch=65535, n_q=1, n_kv=1, heads=1024, kv_heads=1)), ("EINVAL", dict(batch=33, n_kv=1 << 24, heads=1, kv_heads=1)),
    # rows shorter than a token's heads, of half vectors, too long; sequences that overlap
    ("EINVAL", dict(q_row=56)), ("EINVAL", dict(k_row=24)), ("EINVAL", dict(v_row=36)), ("EINVAL", dict(y_row=-64)),
    ("EINVAL", dict(k_row=(1 << 24) + 8)), ("EINVAL", dict(q_batch=5 * 64 - 8)), ("EINVAL", dict(k_batch=9 * 32 - 8)),
    ("EINVAL", dict(v_batch=9 * 32 + 4)), ("EINVAL", dict(y_batch=-8)), ("EINVAL", dict(k_batch=1 << 40)),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("status,over", BAD_GEOM)
def test_geometry_refusals(status, over, backward):
    from paper_2412_02962_amd import pcpp
    assert _status(backward, over) == getattr(pcpp, "PCPP_" + status)
    g = pcpp.make_masked_geom(**{**GEOM, **over})
    assert pcpp.pcpp_masked_attention_workspace_size(g) == 0
    assert pcpp.pcpp_masked_attention_backward_workspace_size(g) == 0


def test_no_geometry():
    from paper_2412_02962_amd import pcpp
    for backward in (False, True):
        assert _status(backward, null_geom=True) == pcpp.PCPP_EINVAL
    assert pcpp.lib().pcpp_masked_attention_workspace_size(None) == 0
    assert pcpp.lib().pcpp_masked_attention_backward_workspace_size(None) == 0


def test_gradients_of_more_queries_than_a_launch_takes():
    from paper_2412_02962_amd import pcpp
    over = dict(batch=9, n_q=1 << 24, n_kv=1, heads=1, kv_heads=1)
    assert _status(True, over) == pcpp.PCPP_EINVAL
    g = pcpp.make_masked_geom(**{**GEOM, **over})
    assert pcpp.pcpp_masked_attention_backward_workspace_size(g) == 0 < pcpp.pcpp_masked_attention_workspace_size(g)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("mask", [
    dict(q_doc=_p("q_doc")), dict(kv_doc=_p("kv_doc")), dict(prefix=_p("prefix")), dict(kv_len=_p("kv_len", 2)),
    dict(q_pos=_p("q_pos", 1)), dict(slopes=_p("slopes", 2)), dict(q_doc=_p("q_doc", 2), kv_doc=_p("kv_doc")),
    # an output, or the workspace, on the mask
    dict(slopes=_p("ws")), dict(kv_len=_p("ws", 4)),
])
def test_mask_refusals(mask, backward):
    from paper_2412_02962_amd import pcpp
    assert _status(backward, mask=mask) == pcpp.PCPP_EINVAL


FORWARD = [
    ("EINVAL", dict(q=None)), ("EINVAL", dict(k=None)), ("EINVAL", dict(v=None)), ("EINVAL", dict(y=None)),
    ("EINVAL", dict(q=_p("q", 8))), ("EINVAL", dict(k=_p("k", 2))), ("EINVAL", dict(v=_p("v", 4))), ("EINVAL", dict(y=_p("y", 8))),
    ("EINVAL", dict(lse=_p("lse", 2))), ("EWORKSPACE", dict(ws=None)), ("EWORKSPACE", dict(wsb=8)),
    ("EINVAL", dict(ws=_p("ws", 8))), ("EINVAL", dict(y=_p("q"))), ("EINVAL", dict(y=_p("k", K_BYTES - 16))),
    ("EINVAL", dict(lse=_p("v"))), ("EINVAL", dict(lse=_p("y"))), ("EINVAL", dict(ws=_p("q", Q_BYTES - 16))),
    ("EINVAL", dict(ws=_p("y"))),
]


@pytest.mark.parametrize("status,over", FORWARD)
def test_forward_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _status(False, **over) == getattr(pcpp, "PCPP_" + status)


BACKWARD = [("EINVAL", {n: None}) for n in ("q", "k", "v", "y", "lse", "dy", "dk", "dv")] + [
    ("EINVAL", {n: _p(n, 8)}) for n in ("q", "k", "v", "y", "dy", "dq", "dk", "dv", "ws")] + [
    ("EINVAL", dict(lse=_p("lse", 2))), ("EINVAL", dict(dq=None, dk=None, dv=None)), ("EWORKSPACE", dict(ws=None)),
    ("EWORKSPACE", dict(wsb=8)), ("EINVAL", dict(dq=_p("q"))), ("EINVAL", dict(dk=_p("k"))), ("EINVAL", dict(dv=_p("dy", 16))),
    ("EINVAL", dict(dq=_p("dy"))), ("EINVAL", dict(dk=_p("lse", 0))),
    ("EINVAL", dict(dk=_p("dv"))), ("EINVAL", dict(dq=_p("dk"))), ("EINVAL", dict(dv=_p("dq"))), ("EINVAL", dict(ws=_p("dq"))), ("EINVAL", dict(ws=_p("y"))),
]


@pytest.mark.parametrize("status,over", BACKWARD)
def test_backward_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _status(True, **over) == getattr(pcpp, "PCPP_" + status)


@pytest.mark.parametrize("backward", [False, True])
def test_the_workspace_holds_to_the_byte(backward):
    from paper_2412_02962_amd import pcpp
    size = pcpp.pcpp_masked_attention_backward_workspace_size if backward else pcpp.pcpp_masked_attention_workspace_size
    need = size(pcpp.make_masked_geom(**GEOM))
    assert _status(backward, wsb=need - 1) == pcpp.PCPP_EWORKSPACE


def test_workspaces():
    from paper_2412_02962_amd import pcpp
    f, b = pcpp.pcpp_masked_attention_workspace_size, pcpp.pcpp_masked_attention_backward_workspace_size
    # the documents' ranges of 64 tokens: 8 bytes each, in units of 16
    assert f(pcpp.make_masked_geom(1, 65, 64, 1, 1, 64)) == 32
    # a token on a long cache: 64 pieces of 8 groups, 32 rows of 128 float32 and two
    assert f(pcpp.make_masked_geom(1, 1, 1 << 20, 32, 8, 128)) == 8 * (1 + (1 << 14)) + 8 + 512 * 32 * 130 * 4
    # two float32 of every query and head
    assert b(pcpp.make_masked_geom(1, 64, 64, 1, 1, 64)) == 16 + 2 * 64 * 4
    # keys' gradients in 18 pieces of the queries, two of 36 tiles each
    assert b(pcpp.make_masked_geom(1, 576, 513, 4, 1, 64, causal=True)) == 8 * (9 + 9) + 2 * 4 * 576 * 4 + 18 * 513 * 2 * 64 * 4
