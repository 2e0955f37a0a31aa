"""Dropout's mask by its definition (include/pcpp.h), and GroupNorm with its
activation and dropout in float64, with how far an implementation may be from
it that computes in float32 and rounds its results once."""

import math

import numpy as np
import torch

F64 = torch.float64
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# act(z) and act'(z): erf to 1.5e-7 and a few float32 roundings (|z| <= 9)
ACT_ERR = 1.5e-6


def philox(block, stream, seed):
    """Philox 4x32-10 of integers, one block."""
    low = 0xFFFFFFFF
    c = [block & low, block >> 32 & low, stream & low, stream >> 32 & low]
    k = [seed & low, seed >> 32 & low]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def kept(n, p, seed, stream, first=0):
    """Which of the elements first .. first + n - 1 are kept (first a multiple of 8)."""
    i = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    stream, seed = stream % 2 ** 64, seed % 2 ** 64
    c = [i & low, i >> half, np.full_like(i, stream & 0xFFFFFFFF), np.full_like(i, stream >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.ascontiguousarray(np.stack(c, -1).astype("<u4")).view("<u2").reshape(-1)[:n]
    return torch.from_numpy(bits >= round(65536 * p))


def factor(p):
    t = round(65536 * p)
    return 0.0 if t == 65536 else 65536 / (65536 - t)


def dropped(v, p, seed, stream):
    if p == 0:
        return v
    keep = kept(v.numel(), p, seed, stream).reshape(v.shape)
    return torch.where(keep, v * factor(p), torch.zeros_like(v))


def act(z, kind):
    """act(z), act'(z), and a bound of |act''|."""
    if kind == "none":
        return z, torch.ones_like(z), 0.0
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s)), 0.5
    phi = 0.5 * (1 + torch.special.erf(z / math.sqrt(2)))
    return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 0.8


def forward(x, gamma, beta, G, eps, kind, p, seed, stream, dtype):
    """A dict of y, mean, rstd and a bound of |y - exact|; x [B, N, C] float64."""
    B, N, C = x.shape
    t = x.reshape(B, N, G, C // G)
    mean = t.mean((1, 3), keepdim=True)
    var = ((t - mean) ** 2).mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    n = ((t - mean) * rstd).reshape(B, N, C)
    z = n * gamma + beta
    a, da, d2 = act(z, kind)
    y = dropped(a, p, seed, stream)
    # float32: the means' merging (a few roundings of values up to the largest),
    # the deviation's difference, and what follows
    top = t.abs().amax((1, 3), keepdim=True)
    e_n = (2.0 ** -20 * (n.abs() + (rstd * (mean.abs() + 0.01 * top)).expand(t.shape).reshape(B, N, C)))
    e_z = e_n * gamma.abs() + 2.0 ** -22 * (z.abs() + beta.abs())
    f = max(factor(p), 1.0)
    bound = HALF[dtype] * y.abs() + f * (e_z * da.abs().clamp(max=1.2) + d2 * e_z ** 2 + (ACT_ERR if kind != "none" else 0)) + 2.0 ** -22 * y.abs() + 1e-30
    return dict(y=y, mean=mean.reshape(B, G), rstd=rstd.reshape(B, G), bound=bound, n=n, z=z, e_n=e_n, e_z=e_z, G=G,
                mean_bound=2.0 ** -20 * (mean.abs() + 0.05 * top).reshape(B, G), rstd_bound=2.0 ** -18 * rstd.reshape(B, G))


def backward(r, gamma, dy, kind, p, seed, stream, dtype):
    """(dx, dgamma, dbeta) from forward()'s dict, and their bounds."""
    B, N, C = dy.shape
    G = r["G"]
    _, da, d2 = act(r["z"], kind)
    d = dropped(dy, p, seed, stream)
    g = d * da
    w, n = g * gamma, r["n"]
    mean = lambda t: t.reshape(B, N, G, C // G).mean((1, 3), keepdim=True).expand(B, N, G, C // G).reshape(B, N, C)
    rstd = r["rstd"][:, None, :, None].expand(B, N, G, C // G).reshape(B, N, C)
    dx = rstd * (w - mean(w) - n * mean(w * n))
    out = dx, (g * n).sum((0, 1)), g.sum((0, 1))
    e_g = d.abs() * (d2 * r["e_z"] + (ACT_ERR if kind != "none" else 0) + 2.0 ** -22)
    e_w = e_g * gamma.abs()
    # sums of M terms in runs, each sum's error a 2^-20th of the quadrature sum
    M = N * (C // G)
    sums = lambda t: 2.0 ** -20 * torch.sqrt(mean(t * t) / M) * math.sqrt(M) / math.sqrt(M) * max(1.0, math.sqrt(M) / 16)
    e0, e1 = mean(e_w) + sums(w), mean(e_w * n.abs() + w.abs() * r["e_n"]) + sums(w * n)
    bx = rstd * (e_w + e0 + n.abs() * e1 + r["e_n"] * mean(w * n).abs() + 2.0 ** -18 * (w.abs() + mean(w).abs() + (n * mean(w * n)).abs()))
    total = lambda t, e: (e).sum((0, 1)) / math.sqrt(B * N) * 6 + 2.0 ** -18 * torch.sqrt((t * t).sum((0, 1)))
    # errors of the terms: those of the formulas may all have one sign
    bg = e_g * n.abs() + g.abs() * r["e_n"]
    bounds = (HALF[dtype] * dx.abs() + bx + 1e-30, 2.0 ** -8 * out[1].abs() + bg.sum((0, 1)) + total(g * n, bg) + 1e-30,
              2.0 ** -8 * out[2].abs() + e_g.sum((0, 1)) + total(g, e_g) + 1e-30)
    return out, bounds
