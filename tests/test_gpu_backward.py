"""GPU tests of the attention backward pass against its plain 64-bit definition (oracle/grad_oracle.py).

Bounds, element by element and derived from the arithmetic:
* P and dS are rounded to BF16 before the second products: half a step, 2^-8 of every term;
* P itself: exp2 by the special-function unit or a cubic (7.5e-5), its argument an fp32 sum of 128 products and two
  more terms (here below 4e-4 in relative error of P): 5e-4 of every term together;
* dP - delta: fp32 sums of 128 products each, 130 * 2^-23 of the sum of magnitudes;
* the outer sums run in fp32 over n terms: n * 2^-23 of the sum of magnitudes (2^-23: the tensor cores may truncate);
* one rounding of the result to BF16: 2^-8 of it.
"""
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import grad_oracle as orc
from paper_2603_24517_b200 import build as lib_build

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


def make(B, Hq, Hkv, Sq, Sk, gain=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * Sq + Sk)

    def t(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    q = (t(B, Sq, Hq, 128) * gain).bfloat16()
    k, v, dout = t(B, Sk, Hkv, 128).bfloat16(), t(B, Sk, Hkv, 128).bfloat16(), t(B, Sq, Hq, 128).bfloat16()
    return dout, q, k, v


def check(got, dout, q, k, v, o, lse, causal, scale, dlse=None):
    want, sizes, noises = orc.attention_grads(dout, q, k, v, o, lse, causal, scale, dlse)
    terms = (k.shape[1], q.shape[1] * (q.shape[2] // k.shape[2]), q.shape[1] * (q.shape[2] // k.shape[2]))
    for name, a, b, size, noise, n in zip(("dq", "dk", "dv"), got, want, sizes, noises, terms):
        a = a.double()
        assert bool(torch.isfinite(a).all()), name
        bound = (2.0 ** -8 + 5e-4 + n * 2.0 ** -23) * size + 130 * 2.0 ** -23 * noise + 2.0 ** -8 * b.abs() + 1e-30
        worst = float(((a - b).abs() / bound).max())
        assert worst <= 1.0, f"{name}: {worst} times the bound"


def grads(dout, q, k, v, causal, scale=SCALE, dlse=None):
    o, lse = lib.attention_forward(q, k, v, causal=causal, scale=scale)
    got = lib.attention_backward(dout, q, k, v, o, lse, causal=causal, scale=scale, dlse=dlse)
    torch.cuda.synchronize()
    assert lib.attn_last_device_status()[0] == 0
    return o, lse, got


SHAPES = [
    (1, 1, 1, 128, 128, False), (1, 1, 1, 128, 128, True), (1, 1, 1, 1, 1, False), (1, 1, 1, 1, 2, True),
    (2, 2, 2, 256, 256, True), (1, 2, 1, 129, 127, False), (1, 4, 2, 127, 257, True), (2, 3, 3, 300, 200, False),
    (1, 2, 2, 300, 77, True), (1, 2, 1, 513, 130, True), (1, 8, 1, 200, 640, True), (1, 8, 8, 1, 1000, True),
    (1, 2, 2, 1000, 1, False), (3, 6, 2, 385, 385, True), (1, 2, 2, 1024, 1024, False), (1, 4, 4, 2048, 2048, True),
    (1, 1, 1, 64, 9000, True), (1, 16, 2, 5, 5, True),
]


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal", SHAPES)
def test_backward_matches_definition(B, Hq, Hkv, Sq, Sk, causal):
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE)
    if causal and Sq > Sk:  # rows without keys
        assert bool((got[0][:, :Sq - Sk] == 0).all())
