"""The 64-bit definitions in oracle/grad_oracle.py, pinned on the CPU: gradients against automatic differentiation and
against central differences of the forward definition, the rotation against complex multiplication."""
import math

import pytest
import torch

from oracle import grad_oracle as orc

D = 16


def _inputs(B, Hq, Hkv, Sq, Sk, seed):
    g = torch.Generator().manual_seed(seed)
    q, dout = (torch.randn(B, Sq, Hq, D, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(B, Sk, Hkv, D, generator=g, dtype=torch.float64) for _ in range(2))
    return dout, q, k, v


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal", [(1, 1, 1, 1, 1, False), (2, 4, 2, 5, 9, True), (1, 3, 1, 9, 5, True),
                                                   (1, 2, 2, 7, 7, False)])
def test_attention_grads_match_autograd_and_differences(B, Hq, Hkv, Sq, Sk, causal):
    dout, q, k, v = _inputs(B, Hq, Hkv, Sq, Sk, 10 * Sq + Sk)
    g = torch.Generator().manual_seed(5)
    dlse = torch.randn(B, Hq, Sq, generator=g, dtype=torch.float64)
    scale = 0.4
    dead = max(0, Sq - Sk) if causal else 0     # rows that see no key: lse = -inf, no gradient through it

    def loss(a, b, c):
        o, lse = orc.attention(a, b, c, causal, scale)
        return (o * dout).sum() + (lse * dlse)[:, :, dead:].sum()

    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    o, lse = orc.attention(*leaves, causal, scale)
    assert bool(torch.isneginf(lse[:, :, :dead]).all()) and bool((o[:, :dead] == 0).all())
    got, sizes, _ = orc.attention_grads(dout, q, k, v, o.detach(), lse.detach(), causal, scale, dlse)
    got = [got[0], got[1], got[2]]
    if not dead:  # logsumexp of an empty row has no usable derivative in autograd
        for a, b in zip(got, torch.autograd.grad(loss(*leaves), leaves)):
            assert torch.allclose(a, b, rtol=1e-9, atol=1e-11)
    eps = 1e-5
    for i in range(3):
        way = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64)
        at = [t.detach() for t in leaves]
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + eps * way, at[i] - eps * way
        slope = (loss(*up) - loss(*down)) / (2 * eps)
        # central differences: third derivative times eps^2 / 6, rounding 1e-16 / eps
        assert math.isclose(float((got[i] * way).sum()), float(slope), rel_tol=1e-6, abs_tol=1e-7)
        assert bool((got[i].abs() <= sizes[i] * (1 + 1e-12) + 1e-15).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [4, 16])
def test_rotation_is_a_complex_product_and_keeps_lengths(interleaved, rot):
    g = torch.Generator().manual_seed(rot)
    x = torch.randn(2, 3, 2, D, generator=g, dtype=torch.float64)
    angle = torch.randn(2, 3, rot // 2, generator=g, dtype=torch.float64)
    y = orc.rotate(x, angle.cos(), angle.sin(), interleaved)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        z = torch.complex(x[..., a], x[..., b]) * torch.exp(1j * angle[:, :, None, i])
        assert torch.allclose(torch.complex(y[..., a], y[..., b]), z, atol=1e-14)
    assert torch.equal(y[..., rot:], x[..., rot:])
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1))


def test_norm_rope_grads_match_differences():
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(2, 3, 2, D, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(D, generator=g, dtype=torch.float64)
    angle = torch.randn(7, 4, generator=g, dtype=torch.float64)
    pos = torch.tensor([[0, 6, 2], [3, 3, 1]])
    args = (angle.cos(), angle.sin(), pos, 1e-6, False)
    dx, dw = orc.norm_rope_grads(dy, x, w, *args)
    eps = 1e-6
    wx, ww = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(D, generator=g, dtype=torch.float64)
    f = lambda a, b: (orc.norm_rope(a, b, *args) * dy).sum()  # noqa: E731
    assert math.isclose(float((dx * wx).sum()), float((f(x + eps * wx, w) - f(x - eps * wx, w)) / (2 * eps)), rel_tol=1e-6)
    assert math.isclose(float((dw * ww).sum()), float((f(x, w + eps * ww) - f(x, w - eps * ww)) / (2 * eps)), rel_tol=1e-6)
