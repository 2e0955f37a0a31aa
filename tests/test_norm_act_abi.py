"""Refusals of dropout and of GroupNorm with its activation: every call here
fails validation before anything would be enqueued."""

import ctypes

import pytest

A = 1 << 24          # an aligned address; never dereferenced
STEP = 1 << 40       # far enough apart for any size used here
NAMES = ("x", "gamma", "beta", "rng", "y", "stats", "dy", "dx", "dgamma", "dbeta", "ws", "residual")


def _p(name, off=0):
    return A + NAMES.index(name) * STEP + off


def _dropout(pcpp, **over):
    a = dict(n=100, x_dtype=pcpp.PCPP_DTYPE_F32, y_dtype=pcpp.PCPP_DTYPE_BF16, p=0.5, rng=_p("rng"), x=_p("x"),
             residual=_p("residual"), y=_p("y"))
    a.update(over)
    return pcpp.lib().pcpp_dropout(a["n"], a["x_dtype"], a["y_dtype"], a["p"], a["rng"], 3, a["x"], a["residual"], a["y"], None)


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(n=0)), ("EINVAL", dict(n=-8)), ("EINVAL", dict(n=(1 << 36) + 1)), ("EINVAL", dict(p=-0.1)),
    ("EINVAL", dict(p=1.5)), ("EINVAL", dict(p=float("nan"))), ("ENOTSUP", dict(x_dtype=9)), ("ENOTSUP", dict(y_dtype=-1)),
    ("EINVAL", dict(x=None)), ("EINVAL", dict(y=None)), ("EINVAL", dict(rng=None)), ("EINVAL", dict(x=_p("x", 8))),
    ("EINVAL", dict(residual=_p("residual", 2))), ("EINVAL", dict(y=_p("y", 4))), ("EINVAL", dict(rng=_p("rng", 4))),
    # x may be replaced where it has y's type, and no other way; the residual too
    ("EINVAL", dict(y=_p("x"))), ("EINVAL", dict(y=_p("x", 16), y_dtype=0)), ("EINVAL", dict(y=_p("residual", 16))),
    ("EINVAL", dict(rng=_p("y", 16))),
])
def test_dropout_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _dropout(pcpp, **over) == getattr(pcpp, "PCPP_" + status)


GEOM = dict(batch=2, tokens=9, channels=64, groups=8, drop=0.1)
BYTES = 2 * 9 * 64 * 2


def _norm(pcpp, backward, geom=None, null=False, wsb=1 << 24, **over):
    g = pcpp.make_norm_act_geom(**{**GEOM, **(geom or {})})
    a = {n: _p(n) for n in NAMES}
    a.update(over)
    gp = None if null else ctypes.byref(g)
    if backward:
        return pcpp.lib().pcpp_group_norm_act_backward(gp, a["x"], a["gamma"], a["beta"], a["stats"], a["rng"], 1, a["dy"],
                                                       a["dx"], a["dgamma"], a["dbeta"], a["ws"], wsb, None)
    return pcpp.lib().pcpp_group_norm_act(gp, a["x"], a["gamma"], a["beta"], a["rng"], 1, a["y"], a["stats"], a["ws"], wsb, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(batch=0)), ("EINVAL", dict(batch=65536)), ("EINVAL", dict(tokens=0)), ("EINVAL", dict(channels=0)),
    ("EINVAL", dict(groups=0)), ("EINVAL", dict(eps=0.0)), ("EINVAL", dict(eps=float("nan"))), ("EINVAL", dict(drop=-0.5)),
    ("EINVAL", dict(drop=1.01)), ("EINVAL", dict(drop=float("nan"))), ("EINVAL", dict(reserved=1)),
    ("ENOTSUP", dict(dtype=5)), ("ENOTSUP", dict(act=3)), ("ENOTSUP", dict(act=-1)), ("ENOTSUP", dict(groups=7)),
    ("ENOTSUP", dict(channels=60, groups=4)), ("EINVAL", dict(batch=1 << 14, tokens=1 << 20)),
])
def test_norm_act_geometry_refusals(status, over, backward):
    from paper_2412_02962_amd import pcpp
    assert _norm(pcpp, backward, over) == getattr(pcpp, "PCPP_" + status)
    assert pcpp.pcpp_group_norm_act_workspace_size(pcpp.make_norm_act_geom(**{**GEOM, **over})) == 0


def test_no_geometry():
    from paper_2412_02962_amd import pcpp
    for backward in (False, True):
        assert _norm(pcpp, backward, null=True) == pcpp.PCPP_EINVAL
    assert pcpp.lib().pcpp_group_norm_act_workspace_size(None) == 0


FORWARD = [("EINVAL", {n: None}) for n in ("x", "gamma", "beta", "y", "rng")] + [
    ("EINVAL", {n: _p(n, 8)}) for n in ("x", "gamma", "beta", "y", "ws")] + [
    ("EINVAL", dict(stats=_p("stats", 2))), ("EINVAL", dict(rng=_p("rng", 4))), ("EWORKSPACE", dict(ws=None)),
    ("EWORKSPACE", dict(wsb=16)), ("EINVAL", dict(y=_p("x", 16))), ("EINVAL", dict(y=_p("x"))), ("EINVAL", dict(stats=_p("y", 32))),
    ("EINVAL", dict(ws=_p("x", BYTES - 16))), ("EINVAL", dict(y=_p("gamma"))), ("EINVAL", dict(ws=_p("rng"))),
]
BACKWARD = [("EINVAL", {n: None}) for n in ("x", "gamma", "beta", "stats", "dy", "dx", "rng")] + [
    ("EINVAL", {n: _p(n, 8)}) for n in ("x", "gamma", "beta", "dy", "dx", "dgamma", "dbeta", "ws")] + [
    ("EINVAL", dict(stats=_p("stats", 2))), ("EWORKSPACE", dict(ws=None)), ("EWORKSPACE", dict(wsb=16)),
    ("EINVAL", dict(dx=_p("x"))), ("EINVAL", dict(dx=_p("dy", 16))), ("EINVAL", dict(dgamma=_p("gamma"))),
    ("EINVAL", dict(dbeta=_p("dgamma", 16))), ("EINVAL", dict(dx=_p("dy"), dgamma=_p("dy", 16))), ("EINVAL", dict(ws=_p("dx"))),
]


@pytest.mark.parametrize("status,over", FORWARD)
def test_norm_act_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _norm(pcpp, False, **over) == getattr(pcpp, "PCPP_" + status)


@pytest.mark.parametrize("status,over", BACKWARD)
def test_norm_act_backward_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _norm(pcpp, True, **over) == getattr(pcpp, "PCPP_" + status)


@pytest.mark.parametrize("backward", [False, True])
def test_the_workspace_holds_to_the_byte(backward):
    from paper_2412_02962_amd import pcpp
    need = pcpp.pcpp_group_norm_act_workspace_size(pcpp.make_norm_act_geom(**GEOM))
    assert need > 0 and _norm(pcpp, backward, wsb=need - 1) == pcpp.PCPP_EWORKSPACE
