"""Plain 64-bit definitions of the gradients and of the per-head norm with rotation (torch double, any device).

Test infrastructure only; shares no code with the CUDA path.  Tensors are [B, S, H, D]; consecutive query heads
share a key head.  ``attention_grads`` also returns what the tests' error bounds are made of.
"""
from __future__ import annotations

import torch


def visible(sq: int, sk: int, causal: bool, device) -> torch.Tensor:
    """[Sq, Sk] truth values: key j is visible to row i iff j <= i + Sk - Sq (causal), else always."""
    if not causal:
        return torch.ones(sq, sk, dtype=torch.bool, device=device)
    i = torch.arange(sq, device=device)[:, None]
    j = torch.arange(sk, device=device)[None, :]
    return j <= i + (sk - sq)


def _heads_first(t):
    return t.double().permute(0, 2, 1, 3)  # [B, H, S, D]


def attention(q, k, v, causal: bool, scale: float):
    """o [B, Sq, Hq, D] and lse [B, Hq, Sq] in 64 bits."""
    g = q.shape[2] // k.shape[2]
    Q = _heads_first(q)
    K, V = (_heads_first(t).repeat_interleave(g, 1) for t in (k, v))
    s = (Q @ K.transpose(-1, -2)) * scale
    s = s.masked_fill(~visible(q.shape[1], k.shape[1], causal, q.device), float("-inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.where(torch.isneginf(s), torch.zeros_like(s), torch.exp(s - lse[..., None]))
    return (p @ V).permute(0, 2, 1, 3), lse


def attention_grads(dout, q, k, v, o, lse, causal: bool, scale: float, dlse=None):
    """(dq, dk, dv) from the definition with the given o and lse, and for each the sum of its terms' magnitudes
    (the size that relative errors of single terms are relative to), and the same sums with P in the place of |dS|
    times the largest row sum |dO| |V| + |dO| |O| (for the absolute errors of dP - delta)."""
    B, Sq, Hq, D = q.shape
    hkv = k.shape[2]
    g = Hq // hkv
    Q, G, O = _heads_first(q), _heads_first(dout), _heads_first(o)
    K, V = (_heads_first(t).repeat_interleave(g, 1) for t in (k, v))
    L = lse.double()[..., None]
    s = (Q @ K.transpose(-1, -2)) * scale
    seen = visible(Sq, k.shape[1], causal, q.device)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isneginf(L), torch.zeros_like(L), L)), torch.zeros_like(s))
    delta = (G * O).sum(-1, keepdim=True)
    if dlse is not None:
        delta = delta - dlse.double()[..., None]
    ds = p * (G @ V.transpose(-1, -2) - delta)
    noise = p * (G.abs() @ V.abs().transpose(-1, -2) + (G * O).abs().sum(-1, keepdim=True))

    def group(t):  # sum over the query heads of a key head
        return t.view(B, hkv, g, t.shape[2], D).sum(2)

    def back(t):
        return t.permute(0, 2, 1, 3)

    grads, sizes, noises = [], [], []
    for x, out in ((ds, grads), (ds.abs(), sizes), (noise, noises)):
        m = (lambda t: t) if out is grads else torch.abs
        out.append(back(x @ m(K)) * scale)
        out.append(back(group(x.transpose(-1, -2) @ m(Q))) * scale)
    grads.append(back(group(p.transpose(-1, -2) @ G)))
    sizes.append(back(group(p.transpose(-1, -2) @ G.abs())))
    noises.append(torch.zeros_like(sizes[-1]))
    return grads, sizes, noises


def rotate(x, cos, sin, interleaved: bool):
    """x [B, S, H, D], cos / sin [B, S, R / 2]: rotates pairs (2 i, 2 i + 1) or (i, i + R / 2) of the first R."""
    half = cos.shape[-1]
    y = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[:, :, None, i], sin[:, :, None, i]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def norm_rope(x, w, cos, sin, positions, eps: float, interleaved: bool):
    """rotate(x / sqrt(mean(x^2) + eps) * w) in 64 bits; positions [B, S] index the tables' rows, w may be None."""
    x = x.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        n = n * w.double()
    return rotate(n, cos.double()[positions], sin.double()[positions], interleaved)


def norm_rope_grads(dy, x, w, cos, sin, positions, eps: float, interleaved: bool):
    """(dx, dw) of sum(dy * norm_rope(x)) by automatic differentiation of the definition above."""
    x = x.detach().double().requires_grad_()
    wd = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.detach().double()
    wd = wd.clone().requires_grad_()
    y = norm_rope(x, wd, cos, sin, positions, eps, interleaved)
    return torch.autograd.grad((y * dy.double()).sum(), (x, wd))
