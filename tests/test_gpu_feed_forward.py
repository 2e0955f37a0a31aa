"""GPU parity of pcpp_gated_ff and pcpp_gated_ff_backward with the float64
reference, element by element, and their use together: on other streams, in
captured graphs, on one workspace, as a chain of a sub-layer's operators.

The bounds (tests/ff_reference.py) are the output's own rounding (half a bf16
step), the independent roundings of the operands that pass through memory in
bf16 (h; [dv, dg] and h), six deviations of their sum, and the float32 sums."""

import pytest
import torch

from tests import ff_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64, BF16, U8 = torch.float64, torch.bfloat16, torch.uint8

# tokens, channels, inner width: single tokens, a few, ragged and whole tiles
# of every size the products use, a long contraction, widths that no tile divides
SHAPES = [(1, 64, 64), (1, 1280, 5120), (2, 640, 2560), (3, 2112, 4160), (5, 64, 8192), (8, 2048, 64), (16, 320, 832),
          (17, 128, 192), (31, 1280, 320), (32, 192, 1088), (33, 640, 704), (64, 64, 128), (77, 704, 1920), (129, 192, 320),
          (200, 2560, 256), (256, 256, 256), (333, 640, 1280), (513, 448, 576), (1025, 128, 512), (2049, 320, 384)]


def _say(*a):
    print("[case]", *a, flush=True)


def _act(kind):
    from paper_2412_02962_amd import pcpp
    return pcpp.PCPP_ACT_SILU if kind == "silu" else pcpp.PCPP_ACT_GELU


def _inputs(M, C, F, seed, bias=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s, k=1.0: (torch.randn(s, generator=gen) * k).to(BF16)
    w = dict(ff1_w=rnd(2 * F, C, k=1.3 * C ** -0.5), ff1_b=rnd(2 * F, k=0.3), ff2_w=rnd(C, F, k=F ** -0.5), ff2_b=rnd(C, k=0.3))
    if not bias:
        w["ff1_b"], w["ff2_b"] = torch.zeros_like(w["ff1_b"]), torch.zeros_like(w["ff2_b"])
    return rnd(M, C), w, rnd(M, C, k=0.05)


def _f64(w):
    return {k: v.to(F64) for k, v in w.items()}


def _dev(w):
    return {k: v.to(DEV) for k, v in w.items()}


def _check(got, want, bound, tag):
    err = (got.cpu().to(F64) - want).abs()
    worst = float((err / bound).max())
    print(f"{tag}: max-abs {float(err.max()):.3e}, worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0, (tag, worst)


class Call:
    """A geometry with its buffers on the device."""

    def __init__(self, M, C, F, kind, w, fill=0xA5, stream=None):
        from paper_2412_02962_amd import pcpp
        self.pcpp, self.stream = pcpp, stream
        self.g, self.wd = pcpp.make_ff_geom(M, C, F, _act(kind)), w
        self.w = pcpp.make_ff_weights(w)
        self.wsb = max(pcpp.pcpp_gated_ff_workspace_size(self.g), pcpp.pcpp_gated_ff_backward_workspace_size(self.g))
        self.ws = torch.full((self.wsb,), fill, dtype=U8, device=DEV)
        self.y, self.dx = torch.empty((M, C), dtype=BF16, device=DEV), torch.empty((M, C), dtype=BF16, device=DEV)
        self.codes = torch.empty((M, 2 * F), dtype=U8, device=DEV)
        self.scales = torch.empty((M, F // 16), dtype=U8, device=DEV)
        self.grads = {k: torch.empty_like(v) for k, v in w.items()}
        self.gp = pcpp.make_ff_grads(self.grads)

    def forward(self, x, kept=True):
        self.pcpp.pcpp_gated_ff(self.g, self.w, x, self.y, self.codes if kept else None, self.scales if kept else None,
                                self.ws, self.wsb, self.stream)

    def backward(self, x, dy, x_scales=None):
        self.pcpp.pcpp_gated_ff_backward(self.g, self.w, x, x_scales, self.codes, self.scales, dy, self.dx, self.gp,
                                         self.ws, self.wsb, self.stream)

    def outputs(self):
        return [self.y, self.codes, self.scales, self.dx] + [self.grads[k] for k in sorted(self.grads)]


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("M,C,F", SHAPES)
def test_forward(M, C, F, kind):
    _say("gated ff", M, C, F, kind)
    x, w, _ = _inputs(M, C, F, 17 * M + C + F)
    c = Call(M, C, F, kind, _dev(w))
    c.forward(x.to(DEV), kept=False)
    torch.cuda.synchronize()
    plain = c.y.clone()
    c.ws.fill_(0x7F)
    c.forward(x.to(DEV))
    torch.cuda.synchronize()
    x, w = x.to(F64), _f64(w)
    pre, _, y = ref.gated_ff(x, w, kind)
    _check(plain, y, ref.gated_ff_bound(x, w, kind), "y")
    _check(c.y, y, ref.gated_ff_bound(x, w, kind), "y with the checkpoint")
    _check(ref.from_8bit(c.codes.cpu(), c.scales.cpu()), pre, ref.pre_bound(x, w), "value and gate in 8 bits")


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("M,C,F", SHAPES)
def test_backward(M, C, F, kind):
    _say("gated ff backward", M, C, F, kind)
    x, w, dy = _inputs(M, C, F, 19 * M + C + F)
    codes, scales = ref.to_8bit(ref.gated_ff(x.to(F64), _f64(w), kind)[0])
    xc, xs = ref.to_8bit(x)
    kept = ref.from_8bit(codes, scales)
    c = Call(M, C, F, kind, _dev(w))
    c.codes, c.scales = codes.to(DEV), scales.to(DEV)
    for eight in (False, True):
        xv = ref.from_8bit(xc, xs) if eight else x.to(F64)
        c.ws.fill_(0xA5)
        if eight:
            c.backward(xc.to(DEV), dy.to(DEV), xs.to(DEV))
        else:
            c.backward(x.to(DEV), dy.to(DEV))
        torch.cuda.synchronize()
        want = ref.gated_ff_backward(xv, _f64(w), kept, dy.to(F64), kind)
        bound = ref.gated_ff_backward_bound(xv, _f64(w), kept, dy.to(F64), kind)
        for k, got in dict(dx=c.dx, **c.grads).items():
            _check(got, want[k], bound[k], f"{k} {'8-bit x' if eight else ''}")


def _check_on_gpu(c, x, dy, kind):
    """Forward and backward against the reference in float64 on the GPU."""
    c.forward(x.to(DEV))
    torch.cuda.synchronize()
    x64, w64, dy64 = x.to(DEV, F64), _f64(c.wd), dy.to(DEV, F64)
    _check(c.y, ref.gated_ff(x64, w64, kind)[2].cpu(), ref.gated_ff_bound(x64, w64, kind).cpu(), "y")
    kept = ref.from_8bit(c.codes.cpu(), c.scales.cpu())
    _check(kept, ref.gated_ff(x64, w64, kind)[0].cpu(), ref.pre_bound(x64, w64).cpu(), "value and gate in 8 bits")
    c.backward(x.to(DEV), dy.to(DEV))
    torch.cuda.synchronize()
    want = ref.gated_ff_backward(x64, w64, kept.to(DEV), dy64, kind)
    bound = ref.gated_ff_backward_bound(x64, w64, kept.to(DEV), dy64, kind)
    for k, t in dict(dx=c.dx, **c.grads).items():
        _check(t, want[k].cpu(), bound[k].cpu(), k)


@pytest.mark.parametrize("M,C,F,tiles", [
    (2570, 1280, 2560, (128, 256)),    # the gate's and its gradient's wide tiles, ragged rows
    (5000, 1344, 2624, (128, 256)),    # and widths that no tile divides
    (4100, 448, 1472, (128, 128)),     # the gradients' square tiles
    (2570, 192, 2368, (128, 128)),     # and in pieces of the contraction
])
def test_wide_tiles(M, C, F, tiles):
    """Sizes whose products run on the wide tiles, forward and backward."""
    from paper_2412_02962_amd import pcpp
    _say("wide tiles", M, C, F)
    kind = "gelu"
    x, w, dy = _inputs(M, C, F, 71)
    c = Call(M, C, F, kind, _dev(w))
    got = [pcpp.pcpp_gated_ff_plan(c.g, k)[0] for k in (pcpp.PCPP_FF_UP, pcpp.PCPP_FF_GATE_GRAD, pcpp.PCPP_FF_X_GRAD)]
    assert got[0] == got[1] == tiles[0] and got[2] == tiles[1], got
    _check_on_gpu(c, x, dy, kind)


@pytest.mark.parametrize("M,C,F,kind", [(2093, 640, 2560, "gelu"), (2570, 320, 1728, "silu"), (4999, 64, 960, "gelu")])
def test_many_small_tiles(M, C, F, kind):
    """The gate's gradient on small tiles, more than two for each of 256 compute units."""
    from paper_2412_02962_amd import pcpp
    _say("many small tiles", M, C, F)
    x, w, dy = _inputs(M, C, F, 73)
    c = Call(M, C, F, kind, _dev(w))
    rows, outputs, _ = pcpp.pcpp_gated_ff_plan(c.g, pcpp.PCPP_FF_GATE_GRAD)
    assert (rows, outputs) == (64, 128) and -(-M // rows) * -(-F // outputs) > 2 * 256
    _check_on_gpu(c, x, dy, kind)


def test_no_biases():
    _say("no biases")
    M, C, F = 70, 128, 192
    x, w, _ = _inputs(M, C, F, 5, bias=False)
    with_zeros = Call(M, C, F, "gelu", _dev(w))
    without = Call(M, C, F, "gelu", {k: v for k, v in _dev(w).items() if k in ("ff1_w", "ff2_w")})
    for c in (with_zeros, without):
        c.forward(x.to(DEV))
    torch.cuda.synchronize()
    for a, b in zip(with_zeros.outputs()[:3], without.outputs()[:3]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("only", ["dx", "ff1_w", "ff1_b", "ff2_w", "ff2_b"])
def test_each_gradient_alone(only):
    """The same bits as with all of them; nothing else is written."""
    from paper_2412_02962_amd import pcpp
    _say("gradient alone", only)
    M, C, F = 150, 192, 320
    x, w, dy = _inputs(M, C, F, 6)
    x, dy, w = x.to(DEV), dy.to(DEV), _dev(w)
    c = Call(M, C, F, "silu", w)
    c.forward(x)
    c.backward(x, dy)
    torch.cuda.synchronize()
    all_of = dict(dx=c.dx.clone(), **{k: v.clone() for k, v in c.grads.items()})
    for t in [c.dx, *c.grads.values()]:
        t.fill_(3.0)
    grads = None if only == "dx" else pcpp.make_ff_grads({only: c.grads[only]})
    c.ws.fill_(0xFF)
    pcpp.pcpp_gated_ff_backward(c.g, c.w, x, None, c.codes, c.scales, dy, c.dx if only == "dx" else None, grads, c.ws, c.wsb)
    torch.cuda.synchronize()
    for k, t in dict(dx=c.dx, **c.grads).items():
        assert torch.equal(t, all_of[k]) if k == only else (t == 3).all(), k


@pytest.mark.parametrize("M", [1, 40, 300])
def test_a_bad_token_stays_alone(M):
    """A NaN token and one of infinities leave the other tokens' outputs, codes
    and dx bit for bit as they were."""
    _say("bad token", M)
    C, F = 128, 256
    x, w, dy = _inputs(M + 2, C, F, 9)
    w, dyd = _dev(w), dy.to(DEV)
    outs = []
    for bad in (False, True):
        t = x.clone()
        if bad:
            t[M // 2], t[M + 1, 5] = float("nan"), float("inf")
        c = Call(M + 2, C, F, "gelu", w)
        c.forward(t.to(DEV))
        c.backward(t.to(DEV), dyd)
        torch.cuda.synchronize()
        outs.append([v.cpu() for v in c.outputs()[:4]])
    keep = [i for i in range(M + 2) if i not in (M // 2, M + 1)]
    for a, b in zip(*outs):
        assert torch.equal(a[keep], b[keep])
    assert outs[1][0][M // 2].isnan().all()


@pytest.mark.parametrize("M,C,F", [(3, 64, 128), (100, 192, 320)])
def test_rows_behind_the_last_stay(M, C, F):
    _say("rows behind", M, C, F)
    x, w, dy = _inputs(M, C, F, 11)
    c = Call(M, C, F, "gelu", _dev(w))
    guards = []

    def guarded(shape, dtype, fill):
        n = shape[0] * shape[1]
        buf = torch.full((n + 4096,), fill, dtype=dtype, device=DEV)
        guards.append((buf, n, fill))
        return buf[:n].view(shape)

    c.y, c.dx = guarded((M, C), BF16, 5.0), guarded((M, C), BF16, 5.0)
    c.codes, c.scales = guarded((M, 2 * F), U8, 99), guarded((M, F // 16), U8, 99)
    c.grads = {k: guarded((v.shape[0], v.numel() // v.shape[0]), BF16, 5.0) for k, v in c.wd.items()}
    c.gp = c.pcpp.make_ff_grads(c.grads)
    wide = torch.full((c.wsb + 4096,), 0x55, dtype=U8, device=DEV)
    guards.append((wide, c.wsb, 0x55))
    c.ws = wide[:c.wsb]
    c.forward(x.to(DEV))
    c.backward(x.to(DEV), dy.to(DEV))
    torch.cuda.synchronize()
    for buf, n, fill in guards:
        assert (buf[n:] == fill).all()


def test_calls_of_all_sizes_on_one_workspace():
    """In one stream, without waiting between: every result is that of a call
    on its own."""
    _say("one workspace")
    shapes = [(300, 320, 640), (1, 640, 2560), (40, 128, 192), (513, 192, 320), (2, 64, 64)]
    calls = []
    for i, (M, C, F) in enumerate(shapes):
        x, w, dy = _inputs(M, C, F, 20 + i)
        calls.append((Call(M, C, F, "silu" if i % 2 else "gelu", _dev(w)), x.to(DEV), dy.to(DEV)))
    want = []
    for c, x, dy in calls:
        c.forward(x)
        c.backward(x, dy)
        torch.cuda.synchronize()
        want.append([t.clone() for t in c.outputs()])
    ws = torch.full((max(c.wsb for c, _, _ in calls),), 0xFF, dtype=U8, device=DEV)
    for c, _, _ in calls:
        c.ws = ws
        for t in c.outputs():
            t.fill_(1)
    torch.cuda.synchronize()
    for _ in range(2):
        for c, x, dy in calls:
            c.forward(x)
            c.backward(x, dy)
    torch.cuda.synchronize()
    for (c, _, _), w in zip(calls, want):
        for a, b in zip(c.outputs(), w):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,C,F", [(1, 640, 2560), (24, 128, 192), (200, 192, 320), (1100, 128, 512)])
def test_captured_and_replayed_on_a_side_stream(M, C, F):
    """Forward and backward in a graph, replayed with eager work and new
    inputs between; every replay against an eager run."""
    _say("graph", M, C, F)
    x, w, dy = _inputs(M, C, F, 31)
    w = _dev(w)
    xs, dys = x.to(DEV), dy.to(DEV)
    side = torch.cuda.Stream()
    c, e = Call(M, C, F, "gelu", w), Call(M, C, F, "gelu", w)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.forward(xs)
        c.backward(xs, dys)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(xs)
        c.backward(xs, dys)
    gen = torch.Generator().manual_seed(1)
    for _ in range(4):
        xs.copy_(torch.randn((M, C), generator=gen).to(BF16))
        for t in c.outputs():
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        e.forward(xs)
        e.backward(xs, dys)
        torch.cuda.synchronize()
        for a, b in zip(c.outputs(), e.outputs()):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Two calls in flight on two streams with a workspace each."""
    _say("two streams")
    M, C, F = 700, 320, 640
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls = []
    for i in range(2):
        x, w, dy = _inputs(M + i, C, F, 41 + i)
        calls.append((Call(M + i, C, F, "gelu", _dev(w)), x.to(DEV), dy.to(DEV)))
    want = []
    for c, x, dy in calls:
        c.forward(x)
        c.backward(x, dy)
        torch.cuda.synchronize()
        want.append([t.clone() for t in c.outputs()])
    for _ in range(5):
        for (c, x, dy), s in zip(calls, streams):
            c.stream = s
            c.forward(x)
            c.backward(x, dy)
    torch.cuda.synchronize()
    for (c, _, _), w in zip(calls, want):
        for a, b in zip(c.outputs(), w):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,C,F", [(1, 128, 192), (90, 320, 640)])
def test_a_sublayer_in_training(M, C, F):
    """s = x + addend, y = RMSNorm(s) in bf16 and 8 bits, branch = FF(y) with
    its checkpoint, and back: each operator against the reference on what the
    one before it left, as a training step runs them."""
    from paper_2412_02962_amd import pcpp
    _say("sub-layer", M, C, F)
    x, w, dout = _inputs(M, C, F, 51)
    gen = torch.Generator().manual_seed(52)
    stream, gamma = torch.randn((M, C), generator=gen) * 3, (1 + 0.2 * torch.randn(C, generator=gen)).to(BF16)
    d_res = torch.randn((M, C), generator=gen) * 0.05
    sd, xd, gd = stream.to(DEV), x.to(DEV), gamma.to(DEV)
    y = torch.empty((M, C), dtype=BF16, device=DEV)
    yc, ys = torch.empty((M, C), dtype=U8, device=DEV), torch.empty((M, C // 32), dtype=U8, device=DEV)
    c = Call(M, C, F, "silu", _dev(w))
    ds, dgamma = d_res.to(DEV), torch.empty_like(gd)
    nb = pcpp.pcpp_rms_norm_backward_workspace_size(M, C)
    nws = torch.empty(nb, dtype=U8, device=DEV)
    doutd = dout.to(DEV)
    pcpp.pcpp_rms_norm(M, C, 1e-6, pcpp.PCPP_DTYPE_F32, sd, xd, gd, sd, y, yc, ys)
    c.forward(y)
    c.backward(yc, doutd, ys)
    pcpp.pcpp_rms_norm_backward(M, C, 1e-6, pcpp.PCPP_DTYPE_F32, sd, gd, c.dx, ds, ds, dgamma, nws, nb)
    torch.cuda.synchronize()
    w64 = _f64(w)
    yv = y.cpu().to(F64)
    assert torch.equal(sd.cpu(), stream + x.float())
    _check(c.y, ref.gated_ff(yv, w64, "silu")[2], ref.gated_ff_bound(yv, w64, "silu"), "branch")
    kept, x8 = ref.from_8bit(c.codes.cpu(), c.scales.cpu()), ref.from_8bit(yc.cpu(), ys.cpu())
    want = ref.gated_ff_backward(x8, w64, kept, dout.to(F64), "silu")
    bound = ref.gated_ff_backward_bound(x8, w64, kept, dout.to(F64), "silu")
    for k, got in dict(dx=c.dx, **c.grads).items():
        _check(got, want[k], bound[k], k)
    want_ds, want_g = ref.rms_norm_backward(sd.cpu().to(F64), gamma.to(F64), c.dx.cpu().to(F64), d_res.to(F64), 1e-6)
    assert torch.allclose(ds.cpu().to(F64), want_ds, rtol=2 ** -20, atol=2 ** -18 * float(want_ds.abs().max()))
    assert torch.allclose(dgamma.cpu().to(F64), want_g, rtol=ref.HALF_BF16, atol=2 ** -18 * float(want_g.abs().max()))
