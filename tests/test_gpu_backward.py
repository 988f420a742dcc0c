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


def check(got, dout, q, k, v, o, lse, causal, scale, dlse=None, operand=2.0 ** -8):
    want, sizes, noises = orc.attention_grads(dout, q, k, v, o, lse, causal, scale, dlse)
    terms = (k.shape[1], q.shape[1] * (q.shape[2] // k.shape[2]), q.shape[1] * (q.shape[2] // k.shape[2]))
    for name, a, b, size, noise, n in zip(("dq", "dk", "dv"), got, want, sizes, noises, terms):
        a = a.double()
        assert bool(torch.isfinite(a).all()), name
        bound = (operand + 5e-4 + n * 2.0 ** -23) * size + 130 * 2.0 ** -23 * noise + 2.0 ** -8 * b.abs() + 1e-30
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


# one key tile and many query tiles, few rows and many keys, and both short: the streams are split and joined
SPLIT_SHAPES = [(1, 1, 1, 128, 8192, False), (1, 2, 1, 64, 9000, True), (1, 8, 2, 5000, 100, False), (2, 4, 4, 1, 4097, True),
                (1, 1, 1, 2048, 2048, True), (1, 4, 1, 2100, 2100, False), (1, 2, 2, 4000, 300, True), (1, 6, 2, 900, 1700, True)]


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal", SPLIT_SHAPES)
def test_split_streams_match_definition(B, Hq, Hkv, Sq, Sk, causal):
    stats = 2 * 4 * B * Hq * ((Sq + 127) // 128 * 128)
    assert lib.attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Sk, 128, causal) > stats   # there are partial sums
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE)
    if causal and Sq > Sk:
        assert bool((got[0][:, :Sq - Sk] == 0).all())


# short query sequences of GQA groups: the group's heads share the rows of a query tile
PACKED_SHAPES = [(1, 8, 1, 1, 1, False), (2, 8, 2, 1, 700, True), (1, 16, 1, 8, 300, True), (1, 16, 1, 9, 300, False),
                 (1, 4, 2, 33, 129, True), (2, 6, 3, 65, 64, True), (1, 8, 1, 130, 130, True), (1, 32, 4, 5, 2500, True),
                 (1, 16, 2, 40, 12, True), (1, 64, 4, 3, 20000, True), (1, 4, 1, 1000, 1000, True), (3, 8, 2, 300, 130, True)]


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal", PACKED_SHAPES)
def test_short_sequences_of_head_groups(B, Hq, Hkv, Sq, Sk, causal):
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk)
    g = torch.Generator(device="cuda").manual_seed(2)
    dlse = torch.randn(B, Hq, Sq, generator=g, device="cuda")
    dead = max(0, Sq - Sk) if causal else 0
    o, lse, got = grads(dout, q, k, v, causal, dlse=dlse)
    dlse[:, :, :dead] = 0
    check(got, dout, q, k, v, o, lse, causal, SCALE, dlse)
    assert bool((got[0][:, :dead] == 0).all())
    # the same on [B, H, S, D] buffers, into slices of larger ones
    big = torch.full((B, Hq + 1, Sq + 3, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    view = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    dq, dk, dv = big[:, :Hq, :Sq].transpose(1, 2), torch.empty_like(k), torch.empty_like(v)
    o2, lse2 = lib.attention_forward(q, k, v, causal=causal, scale=SCALE)
    lib.attn_bwd_strided(view(dout), view(q), view(k), view(v), view(o2), lse2, dq, dk, dv, causal, SCALE, dlse=dlse)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), got))
    assert bool((big[:, Hq] == 7.0).all()) and bool((big[:, :, Sq:] == 7.0).all())


# at most 64 query rows or 64 keys: P and dS are the sum of two BF16 numbers (2^-9 of a term's rounding is rounded to
# half a step again: 2^-16 of the term), so of the operands' roundings next to nothing is left
SHORT_SHAPES = [(1, 1, 1, 1, 1, False), (1, 1, 1, 1, 9, True), (2, 1, 1, 2, 2, True), (1, 4, 2, 169, 3, True), (1, 1, 1, 9, 9, False),
                (1, 8, 2, 1, 34, False), (2, 3, 3, 64, 1000, True), (2, 3, 1, 1000, 64, False), (1, 2, 2, 2000, 37, True),
                (1, 3, 3, 2, 45152, False), (1, 32, 8, 1, 9000, True), (1, 1, 1, 3550, 3, True)]


@pytest.mark.parametrize("gain", [1.0, 4.0])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal", SHORT_SHAPES)
def test_short_sequences_round_results_only(B, Hq, Hkv, Sq, Sk, causal, gain):
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk, gain=gain)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE, operand=2.0 ** -16)


@pytest.mark.parametrize("causal", [False, True])
def test_many_items_per_cta(causal):
    """More items than SMs, of both kinds: CTAs go from item to item, from one kind to the other and back."""
    dout, q, k, v = make(12, 12, 4, 333, 333)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE)


def test_many_rows_without_keys():
    """Whole query tiles see no key: their items have nothing to load, and dq is exactly 0."""
    dout, q, k, v = make(4, 8, 4, 1500, 200)
    o, lse, got = grads(dout, q, k, v, True)
    assert bool(torch.isneginf(lse[:, :, :1300]).all())
    assert bool((got[0][:, :1300] == 0).all())
    check(got, dout, q, k, v, o, lse, True, SCALE)
    # a gradient with respect to lse = -inf says nothing
    dlse = torch.full_like(lse, 3.0)
    o, lse, got = grads(dout, q, k, v, True, dlse=dlse)
    assert bool((got[0][:, :1300] == 0).all())
    check(got, dout, q, k, v, o, lse, True, SCALE, torch.where(torch.isneginf(lse), torch.zeros_like(lse), dlse))


@pytest.mark.parametrize("gain,scale,causal", [(4.0, SCALE, True), (1.0, 0.5, False), (0.01, SCALE, False)])
def test_sharp_and_flat_scores(gain, scale, causal):
    dout, q, k, v = make(1, 4, 2, 700, 700, gain=gain)
    o, lse, got = grads(dout, q, k, v, causal, scale)
    check(got, dout, q, k, v, o, lse, causal, scale)


def test_gradient_with_respect_to_lse():
    dout, q, k, v = make(2, 4, 2, 300, 450)
    g = torch.Generator(device="cuda").manual_seed(9)
    dlse = torch.randn(2, 4, 300, generator=g, device="cuda") * 5
    o, lse, got = grads(dout, q, k, v, True, dlse=dlse)
    check(got, dout, q, k, v, o, lse, True, SCALE, dlse)


def test_gradient_against_differences():
    """The slope of sum(o dout) of the 64-bit forward pass along random directions, by central differences.  The
    bound: each gradient's terms carry at most 2 * 2^-8 + 2^-9 (the two roundings and P's error) of their magnitude, and
    delta is formed from the rounded o, half a step (2^-8) of |dout| |o| in every row."""
    dout, q, k, v = make(1, 2, 1, 150, 200)
    o, lse, got = grads(dout, q, k, v, True)
    _, sizes, noises = orc.attention_grads(dout, q, k, v, o, lse, True, SCALE)
    g = torch.Generator(device="cuda").manual_seed(1)
    eps = 1e-4
    at = [t.double() for t in (q, k, v)]
    for i in range(3):
        way = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + eps * way, at[i] - eps * way
        f = [(orc.attention(*x, True, SCALE)[0] * dout.double()).sum() for x in (up, down)]
        slope = float((f[0] - f[1]) / (2 * eps))
        bound = float((((2.0 ** -7 + 2.0 ** -9) * sizes[i] + 2.0 ** -8 * noises[i]) * way.abs()).sum()) + 1e-5
        assert abs(float((got[i].double() * way).sum()) - slope) <= bound


def _packed(B, S, Hq, Hkv, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(B, S, Hq + 2 * Hkv, 128, generator=g, device="cuda").bfloat16()


def test_strided_views_and_rows_behind_the_end():
    """Slices of a packed projection, a [B, H, S, D] gradient, and outputs inside larger buffers: the same bits as on
    contiguous copies, and nothing else of the buffers is touched."""
    B, S, Hq, Hkv = 2, 260, 4, 2
    qkv = _packed(B, S, Hq, Hkv, 3)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    dout = torch.randn(B, Hq, S, 128, device="cuda").bfloat16().transpose(1, 2)
    qc, kc, vc, dc = (t.contiguous() for t in (q, k, v, dout))
    o, lse = lib.attention_forward(qc, kc, vc, causal=True)
    want = lib.attention_backward(dc, qc, kc, vc, o, lse, causal=True)
    got = lib.attention_backward(dout, q, k, v, o, lse, causal=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    big = torch.full((B, S + 70, Hq + 2 * Hkv, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    dq, dk, dv = big[:, :S, :Hq], big[:, :S, Hq:Hq + Hkv], big[:, :S, Hq + Hkv:]
    lib.attn_bwd_strided(dout, q, k, v, o, lse, dq, dk, dv, True, SCALE)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want))
    assert bool((big[:, S:] == 7.0).all())


def test_split_outputs_on_strided_views():
    dout, q, k, v = make(1, 2, 2, 100, 6000)
    o, lse, want = grads(dout, q, k, v, False)
    bq = torch.full((1, 164, 4, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    bk = torch.full((1, 6100, 5, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    dq, dk, dv = bq[:, 32:132, 1:3], bk[:, :6000, 0:2], bk[:, :6000, 2:4]
    lib.attn_bwd_strided(dout, q, k, v, o, lse, dq, dk, dv, False, SCALE)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want))
    assert bool((bk[:, 6000:] == 7.0).all()) and bool((bk[:, :, 4] == 7.0).all())
    assert bool((bq[:, :32] == 7.0).all()) and bool((bq[:, 132:] == 7.0).all()) and bool((bq[:, :, 0] == 7.0).all())


def test_expanded_gradient_of_a_sum():
    _, q, k, v = make(1, 2, 2, 130, 130)
    o, lse = lib.attention_forward(q, k, v)
    ones = torch.ones((), device="cuda", dtype=torch.bfloat16).expand(q.shape)
    got = lib.attention_backward(ones, q, k, v, o, lse)
    want = lib.attention_backward(torch.ones_like(q), q, k, v, o, lse)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_expanded_gradient_of_a_sum_of_lse():
    dout, q, k, v = make(1, 2, 2, 130, 130)
    o, lse = lib.attention_forward(q, k, v)
    got = lib.attention_backward(dout, q, k, v, o, lse, dlse=torch.ones((), device="cuda").expand(lse.shape))
    want = lib.attention_backward(dout, q, k, v, o, lse, dlse=torch.ones_like(lse))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shape", [(2, 4, 2, 500, 500, True), (1, 2, 2, 64, 9000, False)])
def test_same_bits_every_time_on_any_stream(shape):
    B, Hq, Hkv, Sq, Sk, causal = shape
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk)
    o, lse, want = grads(dout, q, k, v, causal)
    other = make(3, 4, 4, 700, 700, seed=1)
    oo, ol, owant = grads(*other, True)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    results = []
    for r in range(6):
        with torch.cuda.stream(streams[r % 3]):
            results.append((want, lib.attention_backward(dout, q, k, v, o, lse, causal=causal)))
            results.append((owant, lib.attention_backward(other[0], *other[1:], oo, ol, causal=True)))
    torch.cuda.synchronize()
    assert lib.attn_last_device_status()[0] == 0
    for expected, got in results:
        assert all(torch.equal(a, b) for a, b in zip(got, expected))


def test_captured_and_replayed():
    """A captured call, replayed on new inputs; eager calls before, between and after."""
    dout, q, k, v = make(1, 4, 2, 300, 5000)
    o, lse, want = grads(dout, q, k, v, True)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(lib.attn_bwd_workspace_bytes(1, 4, 2, 300, 5000, 128, True), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.attn_bwd(dout, q, k, v, o, lse, dq, dk, dv, True, SCALE, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want))
    new = make(1, 4, 2, 300, 5000, seed=77)
    o2, lse2, want2 = grads(*new, True)
    for dst, src in zip((dout, q, k, v, o, lse), (*new, o2, lse2)):
        dst.copy_(src)
    ws.fill_(255)       # what the workspace holds before does not matter
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want2))


def test_workspace_and_refusals():
    dout, q, k, v = make(1, 2, 2, 200, 200)
    o, lse = lib.attention_forward(q, k, v)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    need = lib.attn_bwd_workspace_bytes(1, 2, 2, 200, 200, 128, False)
    args = (dout, q, k, v, o, lse, dq, dk, dv, False, SCALE)
    assert lib.attn_bwd_status(*args, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")) == 8
    assert lib.attn_bwd_status(*args, workspace=torch.empty(need, dtype=torch.uint8, device="cuda")) == 0
    assert lib.attn_bwd_status(*args, workspace=torch.empty(need + 8, dtype=torch.uint8, device="cuda")[8:]) == 4
    assert lib.attn_bwd_status(dout, q, k, v, o, lse, q, dk, dv, False, SCALE) == 3           # dq is q
    assert lib.attn_bwd_status(dout, q, k, v, o, lse, dq, dk, dk, False, SCALE) == 3          # dv is dk
    with pytest.raises(ValueError):
        lib.attn_bwd(dout.float(), q, k, v, o, lse, dq, dk, dv, False, SCALE)
    with pytest.raises(ValueError):
        lib.attn_bwd(dout, q, k, v, o, None, dq, dk, dv, False, SCALE)
    with pytest.raises(ValueError):
        lib.attn_bwd(dout[:, :100], q, k, v, o, lse, dq, dk, dv, False, SCALE)
    with pytest.raises(lib.AttnError):
        lib.attention_backward(dout, q, k, v, o, lse, scale=float("nan"))
    torch.cuda.synchronize()


def test_explicit_stream_keeps_its_workspace():
    """A call on a stream that is not torch's current one, with a workspace made in the call: memory that the current
    stream allocates and overwrites meanwhile is not that workspace."""
    dout, q, k, v = make(1, 4, 4, 300, 9000)
    o, lse, want = grads(dout, q, k, v, False)
    need = lib.attn_bwd_workspace_bytes(1, 4, 4, 300, 9000, 128, False)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        got = [torch.empty_like(t) for t in (q, k, v)]
        torch.cuda.synchronize()
        lib.attn_bwd(dout, q, k, v, o, lse, *got, False, SCALE, stream=s.cuda_stream)
        for _ in range(4):
            torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_beyond_32_bits():
    """Batch entries 2^31 elements apart (4 GB), for every tensor: the same bits as on contiguous copies."""
    B, S, Hq, Hkv = 2, 150, 2, 1
    dout, q, k, v = make(B, Hq, Hkv, S, S, seed=5)
    o, lse, want = grads(dout, q, k, v, True)
    far = 1 << 31
    buf = torch.empty(far + 16 * S * Hq * 128, device="cuda", dtype=torch.bfloat16)
    at = 0

    def view(t):
        nonlocal at
        out = buf.as_strided(t.shape, (far, *t.stride()[1:]), at)
        at += t[0].numel()
        return out.copy_(t)

    ins = [view(t) for t in (dout, q, k, v, o)]
    outs = [view(torch.zeros_like(t)) for t in (q, k, v)]
    lib.attn_bwd_strided(*ins, lse, *outs, True, SCALE)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
