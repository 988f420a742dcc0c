"""GPU tests of calls on a stream that is not torch's current one, with the workspace made inside the call: memory freed on
the current stream, which a kernel queued there has still to read, is not that workspace."""
import ctypes
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from paper_2603_24517_b200 import build as lib_build

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


def normal(*shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(sum(shape)), device="cuda").bfloat16()


def beside_a_late_reader(need, call, outputs, want):
    """``call(stream)`` while ``need`` bytes that were just freed on the current stream wait there to be read."""
    s = torch.cuda.Stream()
    for _ in range(3):
        for t in outputs:
            t.zero_()
        before = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)  # 50 ms or more: the call is over by then
        after = before.clone()
        del before
        call(s.cuda_stream)
        torch.cuda.synchronize()
        assert bool((after == 7).all())
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
        del after


def test_backward():
    q, k, v, dout = normal(1, 300, 4, 128), normal(1, 9000, 4, 128), normal(1, 9000, 4, 128), normal(1, 300, 4, 128) * 0.5
    o, lse = lib.attention_forward(q, k, v)
    want = lib.attention_backward(dout, q, k, v, o, lse)
    got = [torch.empty_like(t) for t in (q, k, v)]
    need = lib.attn_bwd_workspace_bytes(1, 4, 4, 300, 9000, 128, False)
    beside_a_late_reader(need, lambda s: lib.attn_bwd(dout, q, k, v, o, lse, *got, False, SCALE, stream=s), got, want)
    beside_a_late_reader(need, lambda s: lib.attn_bwd_strided(dout, q, k, v, o, lse, *got, False, SCALE, stream=s), got, want)


def test_rotation_gradient():
    q, k, dq_out, dk_out = normal(2, 50, 4, 128), normal(2, 50, 2, 128), normal(2, 50, 4, 128) * 0.5, normal(2, 50, 2, 128) * 0.5
    w = torch.ones(128, device="cuda")
    angle = torch.arange(50, device="cuda")[:, None] * 1e4 ** (-torch.arange(0, 128, 2, device="cuda") / 128)
    args = (dq_out, dk_out, q, k, w, w, angle.cos(), angle.sin())
    want = lib.qk_norm_rope_backward(*args)
    got = [torch.empty_like(t) for t in want]
    beside_a_late_reader(lib.attn_qk_norm_rope_bwd_workspace_bytes(), lambda s: lib.attn_qk_norm_rope_bwd(*args, *got, stream=s),
                         got, want)


def test_stream_objects():
    q, k, v, dout = normal(1, 65, 2, 128), normal(1, 300, 2, 128), normal(1, 300, 2, 128), normal(1, 65, 2, 128) * 0.5
    o, lse = lib.attention_forward(q, k, v)
    want = lib.attention_backward(dout, q, k, v, o, lse)
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), ctypes.c_void_p(torch.cuda.Stream().cuda_stream), 1, 2):
        got = [torch.zeros_like(t) for t in (q, k, v)]
        torch.cuda.synchronize()
        lib.attn_bwd(dout, q, k, v, o, lse, *got, False, SCALE, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_split_keys():
    q, k, v = normal(1, 8, 2, 128), normal(1, 3000, 2, 128), normal(1, 3000, 2, 128)
    want = [torch.empty_like(q), torch.empty(1, 2, 8, device="cuda")]
    lib.attn_fwd_splitkv(q, k, v, *want, False, SCALE, 4)
    got = [torch.empty_like(t) for t in want]
    need = lib.attn_splitkv_workspace_bytes(1, 2, 8, 128, 4)
    beside_a_late_reader(need, lambda s: lib.attn_fwd_splitkv(q, k, v, *got, False, SCALE, 4, stream=s), got, want)
    s = torch.cuda.Stream()
    got[0].zero_()
    torch.cuda.synchronize()
    lib.attn_fwd_splitkv(q, k, v, *got, False, SCALE, 4, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])
