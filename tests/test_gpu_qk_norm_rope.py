"""GPU tests of the per-head norm with position rotation and its gradient against the plain 64-bit definition.

Bounds, derived from the arithmetic: everything runs in fp32 and is rounded to BF16 once.  Before that rounding a
value is a sum of at most a few products of numbers that carry relative errors of at most 4 * 2^-24 each beside the
sums of 128 squares or products (a tree of at most 12 additions: 12 * 2^-24 of the sum of magnitudes) and rsqrt (2 ulp):
40 * 2^-24 of the sum of the terms' magnitudes covers it, and half a BF16 step is 2^-8 of the value.
Weight gradients are fp32 sums: every one of n terms carries at most 40 * 2^-24, and the longest chain of additions
is bounded by (n + 100) * 2^-24 of the sum of magnitudes.
"""
import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import grad_oracle as orc
from paper_2603_24517_b200 import build as lib_build

pytestmark = pytest.mark.gpu
U = 40 * 2.0 ** -24
HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


def make(B, S, Hq, Hkv, rot, table, weights, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + S)

    def t(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    q, k, dq, dk = (t(B, S, h, 128).bfloat16() for h in (Hq, Hkv, Hq, Hkv))
    w = [None, None] if weights is None else [(1 + 0.3 * t(128)).to(weights) for _ in range(2)]
    angle = t(table, rot // 2).double() * 100
    pos = torch.randint(0, table, (B, S), generator=g, device="cuda")
    return q, k, dq, dk, w, angle.cos().float(), angle.sin().float(), pos


def check_forward(y, x, w, cos, sin, pos, eps, inter):
    want = orc.norm_rope(x, w, cos, sin, pos, eps, inter)
    size = orc.norm_rope(x.abs(), None if w is None else w.abs(), cos.abs(), -sin.abs(), pos, eps, inter).abs() \
        + orc.norm_rope(x.abs(), None if w is None else w.abs(), cos.abs(), sin.abs(), pos, eps, inter).abs()
    bound = U * size + HALF * want.abs()
    assert bool(((y.double() - want).abs() <= bound).all())


def check_backward(dx, dw, dy, x, w, cos, sin, pos, eps, inter):
    want, want_w = orc.norm_rope_grads(dy, x, w, cos, sin, pos, eps, inter)
    xd = x.double()
    r = 1 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + eps)
    g = orc.rotate(dy.double().abs(), cos.double()[pos].abs(), sin.double()[pos].abs(), inter).abs() \
        + orc.rotate(dy.double().abs(), cos.double()[pos].abs(), -sin.double()[pos].abs(), inter).abs()
    gw = g if w is None else g * w.double().abs()
    size = r * (gw + xd.abs() * r * r * (gw * xd.abs()).mean(-1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= U * size + HALF * want.abs()).all())
    if dw is not None:
        terms = g * xd.abs() * r
        n = terms.numel() // 128
        assert bool(((dw.double() - want_w).abs() <= (40 + n + 100) * 2.0 ** -24 * terms.sum((0, 1, 2))).all())


CASES = [  # B, S, Hq, Hkv, rot, interleaved, weights, positions
    (1, 1, 1, 1, 128, False, torch.float32, True), (4, 1, 32, 8, 128, False, torch.bfloat16, True),
    (2, 77, 3, 1, 128, True, torch.bfloat16, True), (1, 130, 16, 16, 64, False, torch.float32, False),
    (3, 33, 9, 17, 32, True, torch.float32, True), (1, 64, 8, 2, 16, False, None, True),
    (2, 257, 5, 5, 96, False, torch.bfloat16, False), (1, 500, 28, 4, 112, True, None, False),
    (64, 1, 7, 1, 80, False, torch.float32, True),
]


@pytest.mark.parametrize("B,S,Hq,Hkv,rot,inter,weights,positions", CASES)
def test_forward_and_backward_match_definition(B, S, Hq, Hkv, rot, inter, weights, positions):
    q, k, dq, dk, w, cos, sin, pos = make(B, S, Hq, Hkv, rot, 1000, weights)
    if not positions:
        pos = torch.arange(S, device="cuda").expand(B, S)
    named = dict(positions=pos if positions else None, eps=1e-5, interleaved=inter)
    y = lib.qk_norm_rope(q, k, w[0], w[1], cos, sin, **named)
    got = lib.qk_norm_rope_backward(dq, dk, q, k, w[0], w[1], cos, sin, **named)
    for i, (x, dy) in enumerate(((q, dq), (k, dk))):
        check_forward(y[i], x, w[i], cos, sin, pos, 1e-5, inter)
        check_backward(got[i], got[2 + i], dy, x, w[i], cos, sin, pos, 1e-5, inter)
        assert (got[2 + i] is None) == (w[i] is None)
