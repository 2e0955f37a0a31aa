"""Refusals of the feed-forward sub-layer's entry points: every call here
fails validation before anything would be enqueued."""

import ctypes

import pytest

A = 1 << 24          # an aligned address; never dereferenced
STEP = 1 << 36       # far enough apart for any size used here


def _p(n):
    return A + n * STEP


def _norm(pcpp, **over):
    a = dict(rows=8, channels=64, eps=1e-6, dtype=pcpp.PCPP_DTYPE_F32, x=_p(0), addend=_p(1), gamma=_p(2), sum_out=_p(3),
             y=_p(4), codes=_p(5), scales=_p(6))
    a.update(over)
    return pcpp.lib().pcpp_rms_norm(a["rows"], a["channels"], a["eps"], a["dtype"], a["x"], a["addend"], a["gamma"],
                                    a["sum_out"], a["y"], a["codes"], a["scales"], None)


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(rows=0)), ("EINVAL", dict(rows=(1 << 24) + 1)), ("EINVAL", dict(channels=0)),
    ("EINVAL", dict(eps=0.0)), ("EINVAL", dict(eps=float("nan"))), ("ENOTSUP", dict(dtype=7)),
    ("ENOTSUP", dict(channels=60)), ("ENOTSUP", dict(channels=8200)), ("ENOTSUP", dict(channels=40)),
    ("EINVAL", dict(x=None)), ("EINVAL", dict(gamma=None)), ("EINVAL", dict(y=None, codes=None, scales=None)),
    ("EINVAL", dict(codes=None)), ("EINVAL", dict(scales=None)), ("EINVAL", dict(x=A + 4)),
    ("EINVAL", dict(codes=_p(5) + 8)), ("EINVAL", dict(y=_p(0))), ("EINVAL", dict(sum_out=_p(1))),
    ("EINVAL", dict(sum_out=_p(0) + 16)), ("EINVAL", dict(codes=_p(4) + 16)), ("EINVAL", dict(scales=_p(5))),
    ("EINVAL", dict(sum_out=_p(0), addend=_p(0) + 32)),
])
def test_rms_norm_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _norm(pcpp, **over) == getattr(pcpp, "PCPP_" + status)


def _norm_backward(pcpp, **over):
    a = dict(rows=8, channels=64, eps=1e-6, dtype=pcpp.PCPP_DTYPE_F32, s=_p(0), gamma=_p(1), dy=_p(2), ds_in=_p(3),
             ds=_p(4), dgamma=_p(5), ws=_p(6), wsb=1 << 20)
    a.update(over)
    return pcpp.lib().pcpp_rms_norm_backward(a["rows"], a["channels"], a["eps"], a["dtype"], a["s"], a["gamma"],
                                             a["dy"], a["ds_in"], a["ds"], a["dgamma"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(rows=0)), ("EINVAL", dict(eps=-1.0)), ("ENOTSUP", dict(dtype=-1)), ("ENOTSUP", dict(channels=12)),
    ("EINVAL", dict(s=None)), ("EINVAL", dict(gamma=None)), ("EINVAL", dict(dy=None)), ("EINVAL", dict(ds=None)),
    ("EWORKSPACE", dict(ws=None)), ("EWORKSPACE", dict(wsb=4)), ("EINVAL", dict(ws=_p(6) + 4)),
    ("EINVAL", dict(dy=_p(2) + 2)), ("EINVAL", dict(ds=_p(0))), ("EINVAL", dict(ds=_p(2))), ("EINVAL", dict(dgamma=_p(1))),
    ("EINVAL", dict(ds_in=_p(4) + 16)), ("EINVAL", dict(ws=_p(4))),
])
def test_rms_norm_backward_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _norm_backward(pcpp, **over) == getattr(pcpp, "PCPP_" + status)


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(rows=0)), ("EINVAL", dict(channels=0)), ("ENOTSUP", dict(channels=48)),
    ("ENOTSUP", dict(channels=65568)), ("ENOTSUP", dict(dtype=2)), ("EINVAL", dict(x=None)), ("EINVAL", dict(codes=None)),
    ("EINVAL", dict(scales=None)), ("EINVAL", dict(x=A + 8)), ("EINVAL", dict(codes=_p(1) + 4)), ("EINVAL", dict(codes=_p(0))),
    ("EINVAL", dict(rows=1 << 24, channels=65536)),
])
def test_checkpoint_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    a = dict(rows=8, channels=64, dtype=pcpp.PCPP_DTYPE_BF16, x=_p(0), codes=_p(1), scales=_p(2))
    a.update(over)
    want = getattr(pcpp, "PCPP_" + status)
    assert pcpp.lib().pcpp_checkpoint_save(a["rows"], a["channels"], a["dtype"], a["x"], a["codes"], a["scales"],
                                           None) == want
    assert pcpp.lib().pcpp_checkpoint_load(a["rows"], a["channels"], a["dtype"], a["codes"], a["scales"], a["x"],
                                           None) == want


GEOMETRIES = [
    ("EINVAL", dict(tokens=0)), ("EINVAL", dict(tokens=-5)), ("EINVAL", dict(tokens=(1 << 24) + 1)),
    ("EINVAL", dict(channels=0)), ("EINVAL", dict(ff_inner=-64)), ("EINVAL", dict(reserved=1)),
    ("EINVAL", dict(tokens=1 << 24, ff_inner=8192)), ("ENOTSUP", dict(channels=96)), ("ENOTSUP", dict(channels=8256)),
    ("ENOTSUP", dict(ff_inner=32)), ("ENOTSUP", dict(ff_inner=65600)), ("ENOTSUP", dict(act=2)), ("ENOTSUP", dict(act=-1)),
]


def _ff(pcpp, g=None, **over):
    g = pcpp.make_ff_geom(**{**dict(tokens=70, channels=128, ff_inner=192), **(g or {})})
    a = dict(ff1_w=_p(0), ff1_b=_p(1), ff2_w=_p(2), ff2_b=_p(3), x=_p(4), y=_p(5), codes=_p(6), scales=_p(7), ws=_p(8),
             wsb=1 << 30)
    a.update(over)
    w = pcpp.make_ff_weights(a)
    return pcpp.lib().pcpp_gated_ff(ctypes.byref(g), ctypes.byref(w), a["x"], a["y"], a["codes"], a["scales"], a["ws"],
                                    a["wsb"], None)


def _ff_backward(pcpp, g=None, **over):
    g = pcpp.make_ff_geom(**{**dict(tokens=70, channels=128, ff_inner=192), **(g or {})})
    a = dict(ff1_w=_p(0), ff1_b=None, ff2_w=_p(2), ff2_b=None, x=_p(4), x_scales=_p(5), codes=_p(6), scales=_p(7),
             dy=_p(8), dx=_p(9), g1=_p(10), gb1=_p(11), g2=_p(12), gb2=_p(13), ws=_p(14), wsb=1 << 30)
    a.update(over)
    w = pcpp.make_ff_weights(a)
    grads = pcpp.pcpp_ff_grads_t(a["g1"], a["gb1"], a["g2"], a["gb2"])
    return pcpp.lib().pcpp_gated_ff_backward(ctypes.byref(g), ctypes.byref(w), a["x"], a["x_scales"], a["codes"],
                                             a["scales"], a["dy"], a["dx"], ctypes.byref(grads), a["ws"], a["wsb"], None)


@pytest.mark.parametrize("status,geom", GEOMETRIES)
def test_gated_ff_geometry(status, geom):
    from paper_2412_02962_amd import pcpp
    want = getattr(pcpp, "PCPP_" + status)
    assert _ff(pcpp, geom) == want and _ff_backward(pcpp, geom) == want
    g = pcpp.make_ff_geom(**{**dict(tokens=70, channels=128, ff_inner=192), **geom})
    assert pcpp.pcpp_gated_ff_workspace_size(g) == 0 and pcpp.pcpp_gated_ff_backward_workspace_size(g) == 0


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(ff1_w=None)), ("EINVAL", dict(ff2_w=None)), ("EINVAL", dict(x=None)), ("EINVAL", dict(y=None)),
    ("EINVAL", dict(codes=None)), ("EINVAL", dict(scales=None)), ("EWORKSPACE", dict(ws=None)), ("EWORKSPACE", dict(wsb=64)),
    ("EINVAL", dict(x=_p(4) + 8)), ("EINVAL", dict(ff2_b=_p(3) + 2)), ("EINVAL", dict(ws=_p(8) + 1)),
    ("EINVAL", dict(y=_p(4))), ("EINVAL", dict(codes=_p(8) + 64)), ("EINVAL", dict(scales=_p(5))), ("EINVAL", dict(ws=_p(2))),
])
def test_gated_ff_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _ff(pcpp, **over) == getattr(pcpp, "PCPP_" + status)


@pytest.mark.parametrize("status,over", [
    ("EINVAL", dict(ff1_w=None)), ("EINVAL", dict(ff2_w=None)), ("EINVAL", dict(x=None)), ("EINVAL", dict(codes=None)),
    ("EINVAL", dict(scales=None)), ("EINVAL", dict(dy=None)), ("EINVAL", dict(dx=None, g1=None, gb1=None, g2=None, gb2=None)),
    ("EWORKSPACE", dict(ws=None)), ("EWORKSPACE", dict(wsb=4096)), ("EINVAL", dict(dy=_p(8) + 4)),
    ("EINVAL", dict(gb1=_p(11) + 2)), ("EINVAL", dict(dx=_p(8))), ("EINVAL", dict(g1=_p(0))), ("EINVAL", dict(g2=_p(10))),
    ("EINVAL", dict(ws=_p(7))), ("EINVAL", dict(dx=_p(5))), ("EINVAL", dict(gb2=_p(14) + 4096)),
])
def test_gated_ff_backward_refusals(status, over):
    from paper_2412_02962_amd import pcpp
    assert _ff_backward(pcpp, **over) == getattr(pcpp, "PCPP_" + status)


def test_null_structs():
    from paper_2412_02962_amd import pcpp
    lib, g = pcpp.lib(), pcpp.make_ff_geom(70, 128, 192)
    assert lib.pcpp_gated_ff_workspace_size(None) == 0 and lib.pcpp_gated_ff_backward_workspace_size(None) == 0
    args = [_p(1), _p(2), None, None, _p(3), 1 << 30, None]
    assert lib.pcpp_gated_ff(None, None, *args) == pcpp.PCPP_EINVAL
    assert lib.pcpp_gated_ff(ctypes.byref(g), None, *args) == pcpp.PCPP_EINVAL


def test_workspace_sizes():
    from paper_2412_02962_amd import pcpp
    for M in (1, 77, 4096):
        g = pcpp.make_ff_geom(M, 640, 2560, pcpp.PCPP_ACT_SILU)
        assert pcpp.pcpp_gated_ff_workspace_size(g) >= 2 * M * 2560
        assert pcpp.pcpp_gated_ff_backward_workspace_size(g) >= 6 * M * 2560 + 2 * M * 640
    assert pcpp.pcpp_rms_norm_backward_workspace_size(100, 640) >= 640 * 4
    assert pcpp.pcpp_rms_norm_backward_workspace_size(0, 640) == 0
    assert pcpp.pcpp_rms_norm_backward_workspace_size(100, 12) == 0


def test_plan():
    """Few tokens straight from memory, few tiles in pieces, many on the largest
    tiles; a plan's queries never need more workspace than the size says."""
    from paper_2412_02962_amd import pcpp
    plan = lambda M, C, F, which: pcpp.pcpp_gated_ff_plan(pcpp.make_ff_geom(M, C, F), which, cus=256)
    assert plan(1, 640, 2560, pcpp.PCPP_FF_UP) == (16, 16, 1)
    assert plan(1, 640, 5120, pcpp.PCPP_FF_UP) == (16, 32, 1)   # 320 workgroups of 16 outputs on 256 units
    assert plan(16, 640, 2560, pcpp.PCPP_FF_DOWN) == (16, 8, 1)
    assert plan(16, 2112, 2560, pcpp.PCPP_FF_DOWN) == (16, 16, 1)
    rows, outputs, pieces = plan(77, 1280, 5120, pcpp.PCPP_FF_DOWN)
    assert rows == 64 and pieces > 1
    assert plan(77, 1280, 5120, pcpp.PCPP_FF_UP)[2] == 1
    assert plan(32768, 1280, 5120, pcpp.PCPP_FF_UP)[0] == 128
    for which in (pcpp.PCPP_FF_W1_GRAD, pcpp.PCPP_FF_W2_GRAD, pcpp.PCPP_FF_X_GRAD):
        assert plan(16384, 1280, 5120, which) == (256, 256, 1)
    assert plan(77, 1280, 5120, pcpp.PCPP_FF_X_GRAD)[2] > plan(77, 1280, 5120, pcpp.PCPP_FF_W1_GRAD)[2] == 1
    for M in (17, 77, 300, 2093):
        for C, F in ((64, 8192), (640, 2560), (1280, 5120)):
            g = pcpp.make_ff_geom(M, C, F)
            pieces = pcpp.pcpp_gated_ff_plan(g, pcpp.PCPP_FF_DOWN, cus=256)[2]
            sums = 4 * M * C * pieces if pieces > 1 else 0
            assert pcpp.pcpp_gated_ff_workspace_size(g) >= 2 * M * F + sums
            need = 6 * M * F + 2 * M * C
            for which, size in ((pcpp.PCPP_FF_W1_GRAD, 2 * F * C), (pcpp.PCPP_FF_W2_GRAD, C * F), (pcpp.PCPP_FF_X_GRAD, M * C)):
                pieces = pcpp.pcpp_gated_ff_plan(g, which, cus=256)[2]
                need += 4 * size * pieces if pieces > 1 else 0
            assert pcpp.pcpp_gated_ff_backward_workspace_size(g) >= need


@pytest.mark.parametrize("which,cus", [(-1, 256), (6, 256), (0, -1)])
def test_plan_refusals(which, cus):
    from paper_2412_02962_amd import pcpp
    with pytest.raises(pcpp.PcppError) as e:
        pcpp.pcpp_gated_ff_plan(pcpp.make_ff_geom(70, 128, 192), which, cus=cus)
    assert e.value.status == pcpp.PCPP_EINVAL
