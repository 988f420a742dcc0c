"""Argument errors of the gradient and rotation entry points, all found before a device is touched."""
import ctypes

import pytest
import torch

import paper_2603_24517_b200 as lib
from paper_2603_24517_b200 import build as lib_build


@pytest.fixture(scope="module")
def cdll():
    lib_build.build()
    return lib.load_library()


def _bwd(c, dout=0x100, q=0x200, k=0x300, v=0x400, o=0x500, lse=0x600, dlse=0, dq=0x700, dk=0x800, dv=0x900, B=1, Hq=2, Hkv=2,
         Sq=128, Sk=128, D=128, causal=0, scale=0.1, ws=0x1000, ws_bytes=1 << 20):
    return c.attn_bwd(dout, q, k, v, o, lse, dlse or None, dq, dk, dv, B, Hq, Hkv, Sq, Sk, D, causal, scale, ws, ws_bytes, None)


def test_backward_argument_errors(cdll):
    for name in ("dout", "q", "k", "v", "o", "lse", "dq", "dk", "dv", "ws"):
        assert _bwd(cdll, **{name: None}) == 1, name
    assert _bwd(cdll, B=0) == 2
    assert _bwd(cdll, Sq=0) == 2
    assert _bwd(cdll, Sk=-1) == 2
    assert _bwd(cdll, Hq=3, Hkv=2) == 2
    assert _bwd(cdll, D=64) == 3
    assert _bwd(cdll, scale=0.0) == 3
    assert _bwd(cdll, scale=float("inf")) == 3
    for name, at in (("dout", 0x108), ("q", 0x208), ("dq", 0x708), ("dk", 0x804), ("dv", 0x902), ("ws", 0x1008), ("lse", 0x602),
                     ("dlse", 0x1601)):
        assert _bwd(cdll, **{name: at}) == 4, name
    assert _bwd(cdll, ws_bytes=100) == 8
    assert _bwd(cdll, dq=0x200) == 3 and _bwd(cdll, dv=0x800) == 3 and _bwd(cdll, ws=0x100) == 3


def test_backward_workspace_size(cdll):
    size = cdll.attn_bwd_workspace_bytes
    stats = lambda B, H, S: 2 * 4 * B * H * ((S + 127) // 128 * 128)  # noqa: E731
    assert size(8, 16, 16, 4096, 4096, 128, 1) == stats(8, 16, 4096)      # enough items: nothing is split
    assert size(1, 2, 2, 512, 512, 128, 0) == stats(1, 2, 512)            # too short to be worth it
    assert size(1, 16, 16, 512, 65536, 128, 1) == stats(1, 16, 512)       # few query items, but they go first
    assert size(1, 1, 1, 64, 9000, 128, 1) > stats(1, 1, 64)              # one query item, a long stream
    assert size(1, 8, 8, 16384, 128, 128, 0) > stats(1, 8, 16384)         # few key items
    # never more than 32 parts of each output
    for a in ((1, 1, 1, 1, 1 << 20), (1, 1, 1, 1 << 20, 1), (1, 8, 1, 100000, 100000)):
        B, Hq, Hkv, Sq, Sk = a
        tiles = B * Hq * ((Sq + 127) // 128) + 2 * B * Hkv * ((Sk + 127) // 128)
        assert size(*a, 128, 0) <= stats(B, Hq, Sq) + 32 * tiles * 65536
    for bad in ((0, 1, 1, 1, 1, 128, 0), (1, 3, 2, 1, 1, 128, 0), (1, 1, 1, 1, 1, 64, 0), (1, 1, 1, 1, 0, 128, 0)):
        assert size(*bad) == 0


def test_backward_stride_errors(cdll):
    arr = lambda *v: (ctypes.c_longlong * 3)(*v)  # noqa: E731
    good = arr(128 * 2 * 128, 2 * 128, 128)

    def call(i=None, s=None):
        st = [good] * 8
        if i is not None:
            st[i] = s
        ptrs = [0x100 * (n + 1) for n in range(6)] + [None] + [0x100 * (n + 7) for n in range(3)]
        return cdll.attn_bwd_strided(*ptrs, 1, 2, 2, 128, 128, 64, *st, 0, 0.1, 0x2000, 1 << 20, None)

    assert call() == 3                       # D = 64, after the strides
    for i in range(8):
        assert call(i, None) == 1
        assert call(i, arr(0, 256, 128)) == 2
        assert call(i, arr(32768, 64, 128)) == 2
        assert call(i, arr(32768, 260, 128)) == 4
        assert call(i, arr(1 << 40, 256, 128)) == 3


def _rope(c, q=0x100, k=0x200, wq=0x300, wk=0x400, wt=0, cos=0x500, sin=0x600, pos=None, pt=0, q_out=0x700, k_out=0x800, B=1,
          S=4, Hq=2, Hkv=1, D=128, rot=128, n=8, inter=0, eps=1e-6, strides=(None,) * 4):
    return c.attn_qk_norm_rope(q, k, wq, wk, wt, cos, sin, pos, pt, None, q_out, k_out, B, S, Hq, Hkv, D, rot, n, inter, eps,
                               *strides, None)


def test_rotation_argument_errors(cdll):
    for name in ("q", "k", "cos", "sin", "q_out", "k_out"):
        assert _rope(cdll, **{name: None}) == 1, name
    for name in ("B", "S", "Hq", "Hkv", "n"):
        assert _rope(cdll, **{name: 0}) == 2, name
    assert _rope(cdll, S=9) == 2                                   # more tokens than positions
    for bad in (dict(D=64), dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(eps=0.0), dict(eps=float("nan")),
                dict(wt=2), dict(pt=-1), dict(B=1 << 30, S=8), dict(q_out=0x200), dict(k_out=0x100), dict(k_out=0x700)):
        assert _rope(cdll, **bad) == 3, bad
    assert _rope(cdll, Hq=2 ** 31 - 1, Hkv=2 ** 31 - 8, S=8) == 3  # head counts at the end of their type
    for name, at in (("q", 0x108), ("wq", 0x304), ("cos", 0x508), ("q_out", 0x708), ("pos", 0x902)):
        assert _rope(cdll, **{name: at}) == 4, name
    assert _rope(cdll, pos=0x904, pt=1) == 4                       # 64-bit positions on a 4-byte address
    arr = lambda *v: (ctypes.c_longlong * 3)(*v)  # noqa: E731
    for i in range(4):
        s = [None] * 4
        s[i] = arr(1024, 100, 128)
        assert _rope(cdll, strides=tuple(s)) == 4                  # not a multiple of 8 elements
        s[i] = arr(1024, 64, 128)
        assert _rope(cdll, strides=tuple(s)) == 2                  # rows would overlap
    assert _rope(cdll, q_out=0x100, strides=(None, None, arr(2048, 512, 128), None)) == 3   # in place, other strides


def _rope_bwd(c, dqo=0x10, dko=0x20, q=0x100, k=0x200, dq=0x700, dk=0x800, dwq=0x900, dwk=0xa00, ws=0x1000, ws_bytes=1 << 20,
              eps=1e-6):
    return c.attn_qk_norm_rope_bwd(dqo, dko, q, k, 0x300, 0x400, 0, 0x500, 0x600, None, 0, None, dq, dk, dwq, dwk, 1, 4, 2, 1,
                                   128, 128, 8, 0, eps, None, None, None, None, None, None, ws, ws_bytes, None)


def test_rotation_gradient_argument_errors(cdll):
    for name in ("dqo", "dko", "q", "k", "dq", "dk", "ws"):
        assert _rope_bwd(cdll, **{name: None}) == 1, name
    assert _rope_bwd(cdll, ws_bytes=cdll.attn_qk_norm_rope_bwd_workspace_bytes() - 1) == 8
    assert _rope_bwd(cdll, eps=-1.0) == 3
    for name, at in (("dqo", 0x18), ("dq", 0x708), ("dwq", 0x902), ("ws", 0x1004)):
        assert _rope_bwd(cdll, **{name: at}) == 4, name
    for bad in (dict(dq=0x200), dict(dq=0x20), dict(dk=0x700), dict(dk=0x100)):
        assert _rope_bwd(cdll, **bad) == 3, bad


def test_cpu_tensors_are_refused():
    q = torch.zeros(1, 4, 2, 128, dtype=torch.bfloat16)
    lse = torch.zeros(1, 2, 4)
    with pytest.raises(ValueError):
        lib.attention_backward(q, q, q, q, q, lse)
    table = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        lib.qk_norm_rope(q, q, None, None, table, table)
    with pytest.raises(ValueError):
        lib.qk_norm_rope_backward(q, q, q, q, None, None, table, table)


def test_workspace_of_a_call_on_the_default_stream(monkeypatch):
    """Stream 0, given as a number, is the default stream, not one out of a pool."""
    from paper_2603_24517_b200 import binding
    recorded, dev = [], torch.device("cuda", 0)

    class Workspace:
        def record_stream(self, stream):
            recorded.append(stream)

    class Like:
        device = dev

        def new_empty(self, n_bytes, dtype):
            return Workspace()

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda stream, device: ("external", stream, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: ("default", device))
    binding._new_workspace(Like(), 64, 0)
    binding._new_workspace(Like(), 64, 0x1230)
    binding._new_workspace(Like(), 64, None)
    assert recorded == [("default", dev), ("external", 0x1230, dev)]
