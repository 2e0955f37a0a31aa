"""Every kind of tile that the feed-forward products run on, with each
activation, whole and in pieces of the contraction: rows, widths and contractions
that no tile divides, against float64.  Each case states the plan it runs on."""

import pytest
import torch

from tests import ff_reference as ref
from tests.test_gpu_feed_forward import Call, _dev, _f64, _inputs

pytestmark = pytest.mark.gpu
DEV, F64 = "cuda", torch.float64

# tokens, channels, inner width: tiles and pieces of the six products, in the
# order PCPP_FF_UP, DOWN, GATE_GRAD, W1_GRAD, W2_GRAD, X_GRAD
UP128, GATE64, GATE128 = (128, 128, 1), (64, 128, 1), (128, 256, 1)


def _square(n, *pieces):
    return [(n, n, k) for k in pieces]


PLANS = {
    (6007, 2112, 448): [UP128, *_square(256, 1), GATE64, *_square(128, 1, 1, 1)],
    (8195, 448, 4160): [UP128, *_square(256, 3), GATE64, *_square(256, 1, 1, 1)],
    (3400, 1280, 5120): [UP128, *_square(256, 3), GATE64, *_square(256, 1, 1, 3)],
    (4099, 448, 5184): [UP128, *_square(128, 3), GATE128, *_square(256, 1, 1, 3)],
    (9999, 448, 1344): [UP128, *_square(128, 1), GATE128, *_square(256, 4, 4, 1)],
    (9999, 192, 2624): [UP128, *_square(128, 1), GATE64, *_square(256, 4, 4, 2)],
    (4100, 448, 1472): [UP128, *_square(128, 1), GATE128, *_square(128, 2, 2, 1)],
    (2570, 192, 2368): [UP128, (64, 128, 1), GATE128, *_square(128, 1, 1, 2)],
}


def _check(got, want, bound, tag):
    worst = float(((got.to(F64) - want).abs() / bound).nan_to_num(float("inf")).max())
    print(f"{tag}: worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0, (tag, worst)


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("M,C,F", list(PLANS))
def test_every_tile(M, C, F, kind):
    from paper_2412_02962_amd import pcpp
    print("[case] tiles", M, C, F, kind, flush=True)
    x, w, dy = _inputs(M, C, F, 83)
    c = Call(M, C, F, kind, _dev(w))
    assert [pcpp.pcpp_gated_ff_plan(c.g, k) for k in range(6)] == PLANS[M, C, F]
    xd, dyd = x.to(DEV), dy.to(DEV)
    c.forward(xd)
    torch.cuda.synchronize()
    x64, w64, dy64 = xd.to(F64), _f64(c.wd), dyd.to(F64)
    _check(c.y, ref.gated_ff(x64, w64, kind)[2], ref.gated_ff_bound(x64, w64, kind), "y")
    kept = ref.from_8bit(c.codes, c.scales)
    _check(kept, ref.gated_ff(x64, w64, kind)[0], ref.pre_bound(x64, w64), "value and gate in 8 bits")
    c.backward(xd, dyd)
    torch.cuda.synchronize()
    want = ref.gated_ff_backward(x64, w64, kept, dy64, kind)
    bound = ref.gated_ff_backward_bound(x64, w64, kept, dy64, kind)
    for k, t in dict(dx=c.dx, **c.grads).items():
        _check(t, want[k], bound[k], k)
