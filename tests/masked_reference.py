"""Masked attention in float64 from its definition (include/pcpp.h), and how
far an implementation may be from it that accumulates in float32 and rounds the
probabilities, the scores' gradients and the results to bf16."""

import math

import torch

F64 = torch.float64
HALF = 2.0 ** -8          # half a step of bf16, relative to the value
SPREAD = 6 / math.sqrt(3)  # six deviations of a uniform rounding, over its half width


class Masks:
    """kv_len [B], q_pos [B], prefix [B], q_doc [B, nq], kv_doc [B, nkv] (int),
    slopes [H] (float); each may be None."""

    def __init__(self, kv_len=None, q_pos=None, prefix=None, q_doc=None, kv_doc=None, slopes=None):
        self.kv_len, self.q_pos, self.prefix = kv_len, q_pos, prefix
        self.q_doc, self.kv_doc, self.slopes = q_doc, kv_doc, slopes


def positions(m, B, nq, nkv, dev):
    first = torch.full((B,), nkv - nq, device=dev) if m.q_pos is None else m.q_pos.to(dev, torch.int64)
    return first[:, None] + torch.arange(nq, device=dev)


def seen(m, B, nq, nkv, causal, dev):
    """[B, nq, nkv], true where the query sees the key."""
    j = torch.arange(nkv, device=dev)[None, None, :]
    ok = torch.ones((B, nq, nkv), dtype=torch.bool, device=dev)
    if m.kv_len is not None:
        ok &= j < m.kv_len.to(dev)[:, None, None]
    if causal:
        past = j <= positions(m, B, nq, nkv, dev)[:, :, None]
        if m.prefix is not None:
            past = past | (j < m.prefix.to(dev)[:, None, None])
        ok &= past
    if m.q_doc is not None:
        qd, kd = m.q_doc.to(dev)[:, :, None], m.kv_doc.to(dev)[:, None, :]
        ok &= (qd == kd) & (qd >= 0)
    return ok


def attention(q, k, v, m, causal=False, scale=None, cap=0.0):
    """q [B, nq, H, D], k, v [B, nkv, KH, D] in float64, finite where seen.
    A dict of y [B, nq, H, D], lse [B, H, nq] and what the bounds take."""
    B, nq, H, D = q.shape
    nkv, KH = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    ok = seen(m, B, nq, nkv, causal, q.device)
    used_k, used_q = ok.any(1), ok.any(2)
    zero = lambda t, used: torch.where(used[:, :, None, None], t, torch.zeros_like(t))
    qh = zero(q, used_q).permute(0, 2, 1, 3)
    kh, vh = (zero(t, used_k).permute(0, 2, 1, 3).repeat_interleave(H // KH, 1) for t in (k, v))
    z = scale * (qh @ kh.transpose(2, 3))
    t = torch.tanh(z / cap) if cap else torch.zeros_like(z)
    s = cap * t if cap else z
    bias = torch.zeros_like(s)
    if m.slopes is not None:
        far = (positions(m, B, nq, nkv, q.device)[:, :, None] - torch.arange(nkv, device=q.device)).abs().to(F64)
        bias = -m.slopes.to(q.device, F64)[None, :, None, None] * far[:, None]
    ok = ok[:, None]
    s = torch.where(ok, s + bias, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.where(ok, torch.exp(s - torch.where(top > -math.inf, top, torch.zeros_like(top))), torch.zeros_like(s))
    total = e.sum(-1, keepdim=True)
    P = e / torch.where(total > 0, total, torch.ones_like(total))
    y = P @ vh
    lse = torch.where(total > 0, top + torch.log(total.clamp(min=1e-300)), torch.full_like(top, -math.inf))[..., 0]
    # of a score: the float32 sum of the product, the transforms' roundings
    mag = 2.0 ** -20 * abs(scale) * torch.sqrt((qh * qh) @ (kh * kh).transpose(2, 3))
    mag = mag + 2.0 ** -21 * (s.abs().nan_to_num(posinf=0) + bias.abs() + 3 * cap + 4 + top.abs().nan_to_num(posinf=0))
    E = torch.where(ok, mag, torch.zeros_like(mag)).amax(-1, keepdim=True)
    return dict(y=y.permute(0, 2, 1, 3), lse=lse, P=P, t=t, E=E, qh=qh, kh=kh, vh=vh, yh=y, scale=scale, KH=KH, cap=cap)


def attention_bound(r, step=HALF):
    """Of |y - exact| and |lse - exact|: y's own rounding; the probabilities'
    (half a step `step`, independent, six deviations of their quadrature sum; in
    the sum that divides them too); the scores'."""
    P, V, y = r["P"], r["vh"], r["yh"]
    through = torch.sqrt((P * P) @ (V * V)) + y.abs() * torch.sqrt((P * P).sum(-1, keepdim=True))
    by = HALF * y.abs() + (SPREAD * step + 2.0 ** -18) * through + 2 * r["E"] * (P @ V.abs() + y.abs()) + 1e-30
    lse = r["lse"]
    bl = SPREAD * step * torch.sqrt((P * P).sum(-1)) + 2 * r["E"][..., 0] + 2.0 ** -21 * lse.abs().nan_to_num(posinf=0)
    return by.permute(0, 2, 1, 3), bl


def gradients(r, dy):
    """dq, dk, dv [B, n, heads, D] from attention()'s dict, and their bounds."""
    B, H, nq, D = r["qh"].shape
    KH, scale, P, t = r["KH"], r["scale"], r["P"], r["t"]
    rows = (P.sum(-1) > 0)[..., None]
    g = torch.where(rows, dy.permute(0, 2, 1, 3), torch.zeros_like(r["qh"]))
    dP = g @ r["vh"].transpose(2, 3)
    delta = (g * r["yh"]).sum(-1, keepdim=True)
    slope = 1 - t * t
    dz = P * (dP - delta) * slope
    shared = lambda x: x.reshape(B, KH, H // KH, *x.shape[2:]).sum(2).permute(0, 2, 1, 3)
    out = dict(dq=scale * (dz @ r["kh"]).permute(0, 2, 1, 3), dk=scale * shared(dz.transpose(2, 3) @ r["qh"]),
               dv=shared(P.transpose(2, 3) @ g))
    # delta takes y as it was rounded; dP is a float32 sum
    by = attention_bound(r)[0].permute(0, 2, 1, 3)
    e_delta = 2 * torch.sqrt((g * g * by * by).sum(-1, keepdim=True)) + 2.0 ** -20 * torch.sqrt((g * g * r["yh"] ** 2).sum(-1, keepdim=True))
    e_dp = 2.0 ** -20 * torch.sqrt((g * g) @ (r["vh"] ** 2).transpose(2, 3))
    ps = P * slope
    E = 3 * r["E"] + 2.0 ** -20
    e_dz = E * dz.abs() + ps * e_dp + 2.0 ** -21 * P * (dP.abs() + delta.abs())  # each, besides delta's
    sq = SPREAD * HALF + 2.0 ** -17
    bq = sq * torch.sqrt((dz * dz) @ r["kh"] ** 2) + e_delta * (ps @ r["kh"]).abs() + e_dz @ r["kh"].abs()
    bk = sq * torch.sqrt((dz * dz).transpose(2, 3) @ r["qh"] ** 2) + e_dz.transpose(2, 3) @ r["qh"].abs()
    bk = bk + 2 * torch.sqrt(((ps * e_delta) ** 2).transpose(2, 3) @ r["qh"] ** 2)
    bv = sq * torch.sqrt((P * P).transpose(2, 3) @ (g * g)) + (E * P).transpose(2, 3) @ g.abs()
    bounds = dict(dq=abs(scale) * bq.permute(0, 2, 1, 3), dk=abs(scale) * shared(bk), dv=shared(bv))
    return out, {n: b + HALF * out[n].abs() + 1e-30 for n, b in bounds.items()}
