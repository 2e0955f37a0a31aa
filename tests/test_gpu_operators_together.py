"""A residual attention block in training, as its calls follow each other:
GroupNorm, SiLU and dropout, masked attention on slices of its output, dropout
with the residual's addition; then the gradients' way back."""

import pytest
import torch

from tests import masked_reference as mref
from tests import norm_act_reference as nref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F64, BF16, F32 = torch.float64, torch.bfloat16, torch.float32
B, N, H, D, G, P, SEED = 2, 333, 4, 40, 8, 0.1, 77
W = H * D            # of the attention
C = 3 * W            # q, k and v side by side
SCALE, CAP = 0.15, 10.0


class Block:
    """Its buffers, allocated once, and its step."""

    def __init__(self, x, skip, gamma, beta, dz, masks):
        from paper_2412_02962_amd import pcpp
        self.lib = pcpp
        self.x, self.skip, self.gamma, self.beta, self.dz = (t.to(DEV) for t in (x, skip, gamma, beta, dz))
        self.masks = {n: t.to(DEV) for n, t in masks.items()}
        self.state = torch.tensor([SEED, 0], dtype=torch.int64, device=DEV)
        empty = lambda *s, t=BF16: torch.empty(s, dtype=t, device=DEV)
        self.qkv, self.dqkv, self.dx = empty(B, N, C), empty(B, N, C), empty(B, N, C)
        self.y, self.dy, self.z = empty(B, N, W), empty(B, N, W), empty(B, N, W)
        self.dgamma, self.dbeta = empty(C), empty(C)
        self.stats, self.lse = empty(B, G, 2, t=F32), empty(B, H, N, t=F32)
        self.norm = pcpp.make_norm_act_geom(B, N, C, G, drop=P)
        self.geom = pcpp.make_masked_geom(B, N, N, H, H, D, causal=True, scale=SCALE, cap=CAP, q_row=C, k_row=C, v_row=C)
        self.bytes = max(pcpp.pcpp_group_norm_act_workspace_size(self.norm), pcpp.pcpp_masked_attention_workspace_size(self.geom),
                         pcpp.pcpp_masked_attention_backward_workspace_size(self.geom))
        self.ws = empty(self.bytes, t=torch.uint8)
        self.outputs = [self.z, self.dx, self.dy, self.dgamma, self.dbeta]

    def step(self):
        p, ws = self.lib, (self.ws, self.bytes)
        m = p.make_mask(**self.masks)
        q, k, v = self.qkv.split(W, -1)
        dq, dk, dv = self.dqkv.split(W, -1)
        bf16 = p.PCPP_DTYPE_BF16
        p.pcpp_group_norm_act(self.norm, self.x, self.gamma, self.beta, self.state, 0, self.qkv, self.stats, *ws)
        p.pcpp_masked_attention(self.geom, m, q, k, v, self.y, self.lse, *ws)
        p.pcpp_dropout(self.y.numel(), bf16, bf16, P, self.state, 1, self.y, self.skip, self.z)
        p.pcpp_dropout(self.y.numel(), bf16, bf16, P, self.state, 1, self.dz, None, self.dy)
        p.pcpp_masked_attention_backward(self.geom, m, q, k, v, self.y, self.lse, self.dy, dq, dk, dv, *ws)
        p.pcpp_group_norm_act_backward(self.norm, self.x, self.gamma, self.beta, self.stats, self.state, 0, self.dqkv, self.dx,
                                       self.dgamma, self.dbeta, *ws)
        self.state[1:].add_(2)


def _inputs():
    gen = torch.Generator().manual_seed(41)
    n = lambda *s: torch.randn(s, generator=gen)
    x, skip, dz = n(B, N, C).to(BF16), n(B, N, W).to(BF16), n(B, N, W).to(BF16)
    gamma, beta = (1.5 + 0.2 * n(C)).to(BF16), (0.2 * n(C)).to(BF16)
    doc = torch.randint(-1, 3, (B, N), generator=gen).sort(-1).values.to(torch.int32)
    masks = dict(q_doc=doc, kv_doc=doc, slopes=2.0 ** -torch.arange(1, H + 1).to(F32), kv_len=torch.tensor([N, N - 50], dtype=torch.int32))
    return x, skip, gamma, beta, dz, masks


def _reference(x, skip, gamma, beta, masks, first):
    """z in float64; largest |score|."""
    t = x.reshape(B, N, G, C // G).transpose(1, 2).reshape(B, G, -1)
    var, mean = torch.var_mean(t, -1, correction=0, keepdim=True)
    t = ((t - mean) / torch.sqrt(var + 1e-5)).reshape(B, G, N, C // G).transpose(1, 2).reshape(B, N, C)
    h = t * gamma + beta
    h = nref.dropped(h * torch.sigmoid(h), P, SEED, first)
    q, k, v = (s.unflatten(-1, (H, D)).transpose(1, 2) for s in h.split(W, -1))
    s = CAP * torch.tanh(SCALE * (q @ k.transpose(2, 3)) / CAP)
    at = torch.arange(N)
    top = float(s.detach().abs().max())
    s = s - masks["slopes"].to(F64)[None, :, None, None] * (at[:, None] - at).abs()
    ok = mref.seen(mref.Masks(**masks), B, N, N, True, "cpu")[:, None]
    # (no exponential of what is hidden: it would spoil the gradient)
    e = torch.where(ok, torch.where(ok, s - torch.where(ok, s, -1e9).amax(-1, keepdim=True).detach(), 0.0).exp(), 0.0)
    total = e.sum(-1, keepdim=True)
    y = (e / torch.where(total > 0, total, 1.0)) @ v
    return skip + nref.dropped(y.transpose(1, 2).flatten(2), P, SEED, first + 1), top


def _far(got, want):
    return float((got.cpu().to(F64) - want).norm() / want.norm())


def test_results_gradients_and_differences():
    x, skip, gamma, beta, dz, masks = _inputs()
    block = Block(x, skip, gamma, beta, dz, masks)
    leaves = [t.to(F64).requires_grad_(True) for t in (x, gamma, beta)]
    for step in range(2):
        block.step()
        torch.cuda.synchronize()
        z, top = _reference(leaves[0], skip.to(F64), *leaves[1:], masks, 2 * step)
        want = torch.autograd.grad(z, leaves, dz.to(F64))
        # Each of the path's ten roundings (the norm's output, P, y, z; dy, dS,
        # delta, P, dqkv, the result) is at most half a step of bf16, relative; the
        # scores' is that of q and k, an exponent's error, twice (P in y and in dS).
        # They are independent: their squares add up.
        bound = (10 + 2 * top ** 2) ** 0.5 * 2.0 ** -8
        assert _far(block.z, z.detach()) <= bound
        for got, w, tag in zip((block.dx, block.dgamma, block.dbeta), want, ("dx", "dgamma", "dbeta")):
            far = _far(got, w)
            print(f"step {step} {tag}: off by {far:.5f} of {bound:.5f}", flush=True)
            assert far <= bound, tag
        # along the gradient: its length against the difference of the whole function
        u = block.dx.cpu().to(F64)
        u = u / u.norm()
        eps = 1e-4
        f = [float((_reference(x.to(F64) + e * u, skip.to(F64), gamma.to(F64), beta.to(F64), masks, 2 * step)[0] * dz.to(F64)).sum())
             for e in (eps, -eps)]
        slope, length = (f[0] - f[1]) / (2 * eps), float((block.dx.cpu().to(F64) * u).sum())
        assert abs(slope - length) <= bound * length


def test_captured_steps():
    """A step in a graph, replayed while another block's steps run eagerly on
    the same stream and a third's on another, each with its own workspace."""
    inputs = _inputs()
    graphed, eager, beside = (Block(*inputs) for _ in range(3))
    graphed.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    eager.step()
    beside.step()
    side = torch.cuda.Stream()
    for step in range(4):
        for t in (graphed, eager, beside):
            t.x.copy_(inputs[0].roll(step, 1))
            for o in t.outputs:
                o.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            beside.step()
        eager.step()
        torch.cuda.synchronize()
        assert int(graphed.state[1]) == int(eager.state[1]) == 2 * (step + 2)
        for a, b, c in zip(graphed.outputs, eager.outputs, beside.outputs):
            assert torch.equal(a, b) and torch.equal(a, c), step
