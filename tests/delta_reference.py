"""The gated delta rule in 64 bits on the CPU, token after token, straight from its definition; gradients by autograd."""
from __future__ import annotations

import torch

from paper_2603_14360_b200 import binding as m


def decay_of(gate, kind, alpha, beta):
    if kind == m.GATE_LOG:
        return torch.exp(gate)
    if kind == m.GATE_LOGIT:
        return torch.sigmoid(gate)
    z = gate + beta
    return torch.exp(-alpha * torch.logaddexp(z, torch.zeros_like(z)))


def one(H, q, k, v, a, b):
    H = H * a[..., None, None]
    u = b[..., None] * (v - torch.einsum("...kv,...k->...v", H, k))
    H = H + torch.einsum("...k,...v->...kv", k, u)
    return H, torch.einsum("...kv,...k->...v", H, q)


def unit(x, eps):
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps)


def prepared(q, k, gate, step, N, o):
    """q, k of every head and the decays and steps; heads are the last but one axis of q and k."""
    if o.get("qk_norm"):
        q, k = unit(q, o["norm_eps"]), unit(k, o["norm_eps"])
    q = q.repeat_interleave(N // q.shape[-2], -2) * o.get("q_scale", 1.0)
    k = k.repeat_interleave(N // k.shape[-2], -2)
    al, be = (None if o.get(x) is None else o[x].double().cpu() for x in ("alpha", "beta"))
    a = decay_of(gate, o.get("gate_kind", m.GATE_LOG), al, be)
    return q, k, a, torch.sigmoid(step) if o.get("step_kind") == m.STEP_LOGIT else step


def scan(q, k, v, gate, step, h0, **o):
    """Dense [B,T,...] tensors in 64 bits -> y, hT."""
    q, k, a, b = prepared(q, k, gate, step, v.shape[2], o)
    H, ys = h0, []
    for t in range(v.shape[1]):
        H, y = one(H, q[:, t], k[:, t], v[:, t], a[:, t], b[:, t])
        ys.append(y)
    return (torch.stack(ys, 1) if ys else torch.zeros_like(v)), H


def scan_any(q, k, v, gate, step, h0, cu=None, **o):
    """scan, or sequence after sequence of a packed batch."""
    if cu is None:
        return scan(q, k, v, gate, step, h0, **o)
    ys, hs = [], []
    for b in range(len(cu) - 1):
        part = [x[cu[b]:cu[b + 1]].unsqueeze(0) for x in (q, k, v, gate, step)]
        y, H = scan(*part, h0[b:b + 1], **o)
        ys.append(y[0])
        hs.append(H)
    return torch.cat(ys), torch.cat(hs)


def gradients(x, h0, dy, d_hT, cu=None, **o):
    """x = (q, k, v, gate, step) and h0 in 64 bits -> y, hT and the gradients of <dy, y> + <d_hT, hT>."""
    leaves = [t.detach().clone().requires_grad_() for t in (*x, h0)]
    y, hT = scan_any(*leaves, cu, **o)
    total = (y * dy).sum() + (0 if d_hT is None else (hT * d_hT).sum())
    g = torch.autograd.grad(total, leaves, allow_unused=True)
    g = [torch.zeros_like(t) if i is None else i for i, t in zip(g, leaves)]
    return y.detach(), hT.detach(), dict(zip(("dq", "dk", "dv", "dgate", "dstep", "dh0"), g))
