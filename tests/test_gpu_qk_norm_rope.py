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


def _contiguous_run(q, k, dq, dk, w, cos, sin, pos, **named):
    y = lib.qk_norm_rope(q.contiguous(), k.contiguous(), *w, cos, sin, positions=pos, **named)
    g = lib.qk_norm_rope_backward(dq.contiguous(), dk.contiguous(), q.contiguous(), k.contiguous(), *w, cos, sin,
                                  positions=pos, **named)
    return y, g


@pytest.mark.parametrize("inter", [False, True])
def test_strided_views_in_place_and_into_a_cache(inter):
    B, S, Hq, Hkv = 2, 51, 6, 2
    _, _, dq, dk, w, cos, sin, pos = make(B, S, Hq, Hkv, 64, 300, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn(B, S, Hq + 2 * Hkv, 128, generator=g, device="cuda").bfloat16()
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    want, wantg = _contiguous_run(q, k, dq, dk, w, cos, sin, pos, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(lib.qk_norm_rope(q, k, *w, cos, sin, positions=pos, interleaved=inter), want))
    # the gradient, written over the incoming gradient
    g1, g2 = dq.clone(), dk.clone()
    dwq, dwk = torch.empty(128, device="cuda"), torch.empty(128, device="cuda")
    lib.attn_qk_norm_rope_bwd(g1, g2, q, k, *w, cos, sin, g1, g2, dwq, dwk, positions=pos, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip((g1, g2, dwq, dwk), wantg))
    # keys into the rows 10 .. 60 of a [B, H, rows, D] cache, the rest of which stays as it is
    cache = torch.full((B, Hkv, 100, 128), 5.0, device="cuda", dtype=torch.bfloat16)
    q_out = torch.empty(B, S, Hq, 128, device="cuda", dtype=torch.bfloat16)
    lib.attn_qk_norm_rope(q, k, *w, cos, sin, q_out, cache.transpose(1, 2)[:, 10:10 + S], positions=pos, interleaved=inter)
    assert torch.equal(cache.transpose(1, 2)[:, 10:10 + S], want[1])
    assert bool((cache[:, :, :10] == 5.0).all()) and bool((cache[:, :, 10 + S:] == 5.0).all())
    # in place, on the slices of the packed projection; the values (v) between them stay
    v = qkv[:, :, Hq + Hkv:].clone()
    lib.attn_qk_norm_rope(q, k, *w, cos, sin, q, k, positions=pos, interleaved=inter)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, Hq + Hkv:], v)


def test_position_types_strides_and_shared_positions():
    B, S = 3, 20
    q, k, dq, dk, w, cos, sin, pos = make(B, S, 4, 2, 128, 500, torch.bfloat16)
    want, wantg = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    wide = torch.zeros(B, 2 * S, device="cuda", dtype=torch.int64)
    wide[:, ::2] = pos
    for p in (pos.int(), wide[:, ::2], pos.t().contiguous().t()):
        got, gotg = _contiguous_run(q, k, dq, dk, w, cos, sin, p)
        assert all(torch.equal(a, b) for a, b in zip(got + gotg, want + wantg))
    row = pos[0].contiguous()
    want, wantg = _contiguous_run(q, k, dq, dk, w, cos, sin, row.expand(B, S).contiguous())
    for p in (row, row.expand(B, S), row.int()):
        got, gotg = _contiguous_run(q, k, dq, dk, w, cos, sin, p)
        assert all(torch.equal(a, b) for a, b in zip(got + gotg, want + wantg))


def test_positions_outside_the_tables_make_nan_rows():
    q, k, dq, dk, w, cos, sin, pos = make(2, 9, 3, 2, 64, 50, torch.float32)
    bad = pos.clone()
    bad[0, 3], bad[1, 8], bad[1, 0] = 50, -1, 1 << 40
    out = torch.zeros(2, 9, dtype=torch.bool, device="cuda")
    out[0, 3] = out[1, 8] = out[1, 0] = True
    y = lib.qk_norm_rope(q, k, *w, cos, sin, positions=bad)
    good = lib.qk_norm_rope(q, k, *w, cos, sin, positions=pos)
    g = lib.qk_norm_rope_backward(dq, dk, q, k, *w, cos, sin, positions=bad)
    for a, b in zip(y, good):
        assert bool(torch.isnan(a[out]).all()) and torch.equal(a[~out], b[~out])
    assert bool(torch.isnan(g[0][out]).all()) and bool(torch.isfinite(g[0][~out]).all())
    assert bool(torch.isnan(g[2]).all())


def test_infinities_and_nan_stay_in_their_rows():
    q, k, dq, dk, w, cos, sin, pos = make(1, 12, 3, 3, 128, 50, torch.float32)
    want = lib.qk_norm_rope(q, k, *w, cos, sin, positions=pos)
    q2 = q.clone()
    q2[0, 5, 1, 7], q2[0, 2, 0, 100] = float("inf"), float("nan")
    y = lib.qk_norm_rope(q2, k, *w, cos, sin, positions=pos)
    keep = torch.ones(1, 12, 3, dtype=torch.bool, device="cuda")
    keep[0, 5, 1] = keep[0, 2, 0] = False
    assert torch.equal(y[0][keep], want[0][keep]) and torch.equal(y[1], want[1])
    assert not bool(torch.isfinite(y[0][~keep]).all())


def test_rows_of_zeros_and_of_large_and_small_values():
    q, k, dq, dk, w, cos, sin, pos = make(1, 40, 4, 4, 128, 50, torch.float32)
    q[:, 0] = 0
    q[:, 1] *= 1e15
    q[:, 2] *= 1e-3
    y = lib.qk_norm_rope(q, k, *w, cos, sin, positions=pos)
    g = lib.qk_norm_rope_backward(dq, dk, q, k, *w, cos, sin, positions=pos)
    assert bool((y[0][:, 0] == 0).all())
    check_forward(y[0], q, w[0], cos, sin, pos, 1e-6, False)
    check_backward(g[0], g[2], dq, q, w[0], cos, sin, pos, 1e-6, False)


def test_same_bits_on_any_stream_and_in_a_graph():
    q, k, dq, dk, w, cos, sin, pos = make(4, 300, 8, 2, 128, 1000, torch.bfloat16)
    want, wantg = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    got2 = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    torch.cuda.synchronize()
    for a, b in ((got, want), (got2, want)):
        assert all(torch.equal(x, y) for x, y in zip(a[0] + a[1], want + wantg))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    q.copy_(q.flip(0))
    pos.copy_(pos.flip(0))
    want, wantg = _contiguous_run(q, k, dq, dk, w, cos, sin, pos)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(cap[0] + cap[1], want + wantg))


def test_offsets_beyond_32_bits():
    """Rows, positions and table rows more than 2^31 elements into their tensors."""
    B, S, Hq, Hkv = 2, 9, 3, 2
    q, k, dq, dk, w, _, _, _ = make(B, S, Hq, Hkv, 128, 16, torch.float32)
    far = 1 << 31
    table = far // 64 + 100
    cos, sin = torch.zeros(table, 64, device="cuda"), torch.zeros(table, 64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    angle = torch.randn(50, 64, generator=g, device="cuda")
    cos[-50:], sin[-50:] = angle.cos(), angle.sin()
    near = torch.randint(0, 50, (B, S), generator=g, device="cuda")
    want, wantg = _contiguous_run(q, k, dq, dk, w, angle.cos().contiguous(), angle.sin().contiguous(), near)
    buf = torch.empty(far + 64 * S * Hq * 128, device="cuda", dtype=torch.bfloat16)
    at = 0

    def view(t):
        nonlocal at
        out = buf.as_strided(t.shape, (far, *t.stride()[1:]), at)
        at += t[0].numel()
        return out.copy_(t)

    qv, kv, dqv, dkv, q_out, k_out = (view(t) for t in (q, k, dq, dk, q, k))
    pos = near + (table - 50)
    lib.attn_qk_norm_rope(qv, kv, *w, cos, sin, q_out, k_out, positions=pos)
    dwq, dwk = torch.empty(128, device="cuda"), torch.empty(128, device="cuda")
    lib.attn_qk_norm_rope_bwd(dqv, dkv, qv, kv, *w, cos, sin, dqv, dkv, dwq, dwk, positions=pos)
    torch.cuda.synchronize()
    assert torch.equal(q_out, want[0]) and torch.equal(k_out, want[1])
    assert all(torch.equal(a, b) for a, b in zip((dqv, dkv, dwq, dwk), wantg))


def test_refusals():
    q, k, dq, dk, w, cos, sin, pos = make(1, 8, 2, 2, 128, 16, torch.float32)
    out = (torch.empty_like(q), torch.empty_like(k))
    ok = lambda *a, **n: lib.attn_qk_norm_rope_status(*a, **n)  # noqa: E731
    assert ok(q, k, *w, cos, sin, *out) == 0
    assert ok(q, k, *w, cos, sin, *out, eps=0.0) == 3
    assert ok(q, k, *w, cos[:, :4].contiguous(), sin[:, :4].contiguous(), *out) == 3        # rot_dim 8
    assert ok(q, k, *w, cos[:7].contiguous(), sin[:7].contiguous(), *out) == 2              # 8 tokens, 7 positions
    assert ok(q, k, *w, cos, sin, out[0], out[0]) == 3                                      # one output for both
    assert ok(q, k, *w, cos, sin, k, out[1]) == 3                                           # queries over keys
    turned = torch.as_strided(q, q.shape, (q.stride(0), 128, 8 * 128, 1))
    assert ok(q, k, *w, cos, sin, turned, out[1]) == 3                                      # in place, other strides
    for bad in (dict(positions=pos.float()), dict(positions=pos[:, :4])):
        with pytest.raises(ValueError):
            ok(q, k, *w, cos, sin, *out, **bad)
    with pytest.raises(ValueError):
        ok(q.float(), k, *w, cos, sin, *out)
    with pytest.raises(ValueError):
        ok(q, k, w[0], w[1].bfloat16(), cos, sin, *out)
    with pytest.raises(ValueError):
        ok(q, k[:, :, :, :64], *w, cos, sin, *out)
    with pytest.raises(ValueError):
        ok(q, k, *w, cos.double(), sin, *out)
    torch.cuda.synchronize()


def test_layer_step_with_attention():
    """Projection slices -> norm and rotation -> attention -> its gradient -> the gradient of norm and rotation, queued
    without a wait in between, in a graph too; every stage against its definition on what the stage before left."""
    B, S, Hq, Hkv = 2, 270, 8, 2
    g = torch.Generator(device="cuda").manual_seed(8)
    qkv = torch.randn(B, S, Hq + 2 * Hkv, 128, generator=g, device="cuda").bfloat16()
    dout = torch.randn(B, S, Hq, 128, generator=g, device="cuda").bfloat16()
    _, _, _, _, w, cos, sin, _ = make(B, S, Hq, Hkv, 128, 400, torch.float32)
    pos = torch.arange(S, device="cuda") + torch.tensor([[0], [100]], device="cuda")

    def step():
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:].contiguous()
        qr, kr = lib.qk_norm_rope(q, k, *w, cos, sin, positions=pos)
        o, lse = lib.attention_forward(qr, kr, v, causal=True)
        dqr, dkr, dv = lib.attention_backward(dout, qr, kr, v, o, lse, causal=True)
        dq, dk, dwq, dwk = lib.qk_norm_rope_backward(dqr, dkr, q, k, *w, cos, sin, positions=pos)
        return q, k, v, qr, kr, o, lse, dqr, dkr, dv, dq, dk, dwq, dwk

    from test_gpu_backward import SCALE, check
    first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first[3:], captured[3:]))
    q, k, v, qr, kr, o, lse, dqr, dkr, dv, dq, dk, dwq, dwk = first
    for x, y, dy, dx, dw, wt in ((q, qr, dqr, dq, dwq, w[0]), (k, kr, dkr, dk, dwk, w[1])):
        check_forward(y, x, wt, cos, sin, pos, 1e-6, False)
        check_backward(dx, dw, dy, x, wt, cos, sin, pos, 1e-6, False)
    check((dqr, dkr, dv), dout, qr, kr, v, o, lse, True, SCALE)
