"""The feed-forward sub-layer's operators in float64 on the CPU, from their
definitions (include/pcpp.h), and how far a float32-accumulating bf16
implementation may be from them."""

import math

import torch

GROUP, MIN_EXP = 32, -117
F64 = torch.float64
# Half a step, relative to the value: bf16 (7 stored mantissa bits), e4m3 (3).
HALF_BF16, HALF_E4M3 = 2.0 ** -8, 2.0 ** -4
# erf to 1.5e-7 (the formula's own bound) and a few float32 roundings, of
# gates up to 8: act(g) and act'(g) are off by less than this.
ACT_ERR = 1.5e-6


def scale_exponents(v):
    """e of every group: the smallest integer >= -117 with max |v| / 2^e <= 448."""
    a = v.to(F64).reshape(v.shape[0], -1, GROUP)
    top = torch.where(torch.isfinite(a), a.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)                       # top = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(top > 0, e, torch.full_like(e, MIN_EXP)).clamp(min=MIN_EXP)


def to_8bit(v):
    """(codes, scales) of rows; the code is chosen in float64."""
    e = scale_exponents(v)
    t = torch.ldexp(v.to(F64).reshape(*e.shape, GROUP), -e[..., None])
    a = t.abs()
    _, k = torch.frexp(a)                         # a in [2^(k-1), 2^k)
    step = torch.exp2((k - 1).clamp(min=-6).to(F64) - 3)
    q = torch.round(a / step) * step              # ties to even
    fin = torch.isfinite(t)
    q = torch.where(fin, q, 0.0)
    # q = (1 + man / 8) 2^(exp - 7), or man 2^-9 below 2^-6
    _, k = torch.frexp(q)
    ex = torch.where(q >= 2.0 ** -6, k - 1 + 7, 0)
    man = torch.where(q >= 2.0 ** -6, (q / torch.exp2((k - 1).to(F64)) - 1) * 8, q * 512)
    code = (ex * 8 + man.to(torch.int64)) + torch.where(torch.signbit(t), 128, 0)
    code = torch.where(fin, code, 127)
    return code.to(torch.uint8).reshape(v.shape), (e + 127).to(torch.uint8)


def from_8bit(codes, scales):
    c = codes.to(torch.int64).reshape(*scales.shape, GROUP)
    ex, man = (c >> 3) & 15, (c & 7).to(F64)
    mag = torch.where(ex == 0, man * 2.0 ** -9, (1 + man / 8) * torch.exp2(ex.to(F64) - 7))
    mag = torch.where((c & 127) == 127, torch.full_like(mag, float("nan")), mag)
    val = torch.where(c >= 128, -mag, mag) * torch.exp2(scales.to(F64) - 127)[..., None]
    return val.reshape(codes.shape)


def act(g, kind):
    """act(g), act'(g)."""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    phi = 0.5 * (1 + torch.special.erf(g / math.sqrt(2)))
    return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def rms_norm(s, gamma, eps):
    return s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * gamma


def rms_norm_backward(s, gamma, dy, ds_in, eps):
    r = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    n, w = s * r, dy * gamma
    ds = r * (w - n * (w * n).mean(-1, keepdim=True))
    return (ds if ds_in is None else ds + ds_in), (dy * n).sum(0)


def gated_ff(x, w, kind):
    """(pre, h, y)."""
    F = w["ff2_w"].shape[1]
    pre = x @ w["ff1_w"].t() + w["ff1_b"]
    h = pre[:, :F] * act(pre[:, F:], kind)[0]
    return pre, h, h @ w["ff2_w"].t() + w["ff2_b"]


def gated_ff_backward(x, w, pre, dy, kind):
    """dict of dx and the gradients, from v and g as they were kept."""
    F = w["ff2_w"].shape[1]
    v, (a, da) = pre[:, :F], act(pre[:, F:], kind)
    dh = dy @ w["ff2_w"]
    dpre = torch.cat([dh * a, dh * v * da], 1)
    return dict(dx=dpre @ w["ff1_w"], ff1_w=dpre.t() @ x, ff1_b=dpre.sum(0), ff2_w=dy.t() @ (v * a), ff2_b=dy.sum(0))


def _through(err, mag, other):
    """Bound of sum_k e_k other_k: `err` bounds each e_k (added up as they
    are), `mag` the values whose bf16 rounding the product sees: independent,
    mean zero, variance at most (half a step)^2 / 3; six deviations, and the
    float32 sum's own."""
    dev = torch.sqrt((mag * mag) @ (other * other))
    return err @ other.abs() + (6 / math.sqrt(3) * HALF_BF16 + 2.0 ** -17) * dev


def gated_ff_bound(x, w, kind):
    """Elementwise bound of |y - exact|."""
    pre, h, y = gated_ff(x, w, kind)
    F = h.shape[1]
    e_pre = 2.0 ** -19 * torch.sqrt((x * x) @ (w["ff1_w"] * w["ff1_w"]).t()) + 2.0 ** -23 * pre.abs()
    a, da = act(pre[:, F:], kind)
    e_h = e_pre[:, :F] * a.abs() + pre[:, :F].abs() * (ACT_ERR + e_pre[:, F:] * da.abs())
    return HALF_BF16 * y.abs() + _through(e_h, h, w["ff2_w"].t()) + 1e-9


def pre_bound(x, w):
    """Bound of |8-bit v, g read back - exact|, with the exact group's scale:
    half a code's step, and the float32 sum's error, which may also move the
    value (or its group's largest) over a border: one step in place of half."""
    pre, _, _ = gated_ff(x, w, "silu")
    e = torch.exp2(scale_exponents(pre).to(F64)).repeat_interleave(GROUP, 1)
    err = 2.0 ** -19 * torch.sqrt((x * x) @ (w["ff1_w"] * w["ff1_w"]).t()) + 2.0 ** -23 * pre.abs()
    return torch.maximum(HALF_E4M3 * pre.abs(), 2.0 ** -10 * e) * (1 + 2.0 ** -10) + 2 * err


def gated_ff_backward_bound(x, w, pre, dy, kind):
    F = w["ff2_w"].shape[1]
    v, (a, da) = pre[:, :F], act(pre[:, F:], kind)
    dh = dy @ w["ff2_w"]
    e_dh = 2.0 ** -19 * torch.sqrt((dy * dy) @ (w["ff2_w"] * w["ff2_w"])) + 2.0 ** -23 * dh.abs()
    dpre = torch.cat([dh * a, dh * v * da], 1)
    e_dpre = torch.cat([e_dh * a.abs() + dh.abs() * ACT_ERR, v.abs() * (e_dh * da.abs() + dh.abs() * ACT_ERR)], 1)
    g = gated_ff_backward(x, w, pre, dy, kind)
    half = lambda k: HALF_BF16 * g[k].abs() + 1e-9
    M = x.shape[0]
    sums = lambda t: 2.0 ** -22 * math.sqrt(M) * torch.sqrt((t * t).sum(0))
    return dict(dx=half("dx") + _through(e_dpre, dpre, w["ff1_w"]),
                ff1_w=half("ff1_w") + _through(e_dpre.t(), dpre.t(), x),
                ff1_b=half("ff1_b") + e_dpre.sum(0) + sums(dpre),
                ff2_w=half("ff2_w") + _through(v.abs().t() * ACT_ERR, (v * a).t(), dy).t(),
                ff2_b=half("ff2_b") + sums(dy))
