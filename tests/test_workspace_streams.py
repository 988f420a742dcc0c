"""Which stream's memory a workspace made inside a call comes from.  On the CPU, with the stream calls of torch recorded: an
allocation while another stream is current could return memory that kernels queued there still use."""
import contextlib

import pytest
import torch

from paper_2603_24517_b200 import binding

DEV = torch.device("cuda", 0)


@pytest.fixture
def made(monkeypatch):
    """The stream that was current at each allocation (None: torch's own choice)."""
    seen, current = [], [None]

    class Workspace:
        def record_stream(self, stream):
            pass

    class Like:
        device = DEV

        def new_empty(self, n_bytes, dtype):
            seen.append(current[-1])
            return Workspace()

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda stream, device: ("external", stream, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: ("default", device))
    return Like(), seen


def test_workspace_comes_from_the_stream_of_the_call(made):
    like, seen = made
    binding._new_workspace(like, 64, 0x1230)
    binding._new_workspace(like, 64, 0)
    binding._new_workspace(like, 64, None)
    assert seen == [("external", 0x1230, DEV), ("default", DEV), None]


def test_every_form_of_a_stream(made):
    """What ctypes passes on as a cudaStream_t, as the other entry points take it."""
    import ctypes
    like, seen = made

    class Stream:
        cuda_stream = 0x1230

    for form in (Stream(), ctypes.c_void_p(0x1230), 2):   # 2: the calling thread's default stream
        binding._new_workspace(like, 64, form)
    assert seen == [("external", 0x1230, DEV)] * 2 + [("external", 2, DEV)]
    del seen[:]
    for form in (1, ctypes.c_void_p(0), ctypes.c_void_p(1)):
        binding._new_workspace(like, 64, form)
    assert seen == [("default", DEV)] * 3


def test_split_keys_make_their_workspace_there_too(monkeypatch):
    made, calls = [], []

    class Lib:
        def attn_splitkv_workspace_bytes(self, *sizes):
            return 4096

        def attn_fwd_splitkv(self, *args):
            calls.append(args)
            return 0

    q = torch.zeros(1, 2, 2, 128, dtype=torch.bfloat16)
    monkeypatch.setattr(binding, "load_library", Lib)
    monkeypatch.setattr(binding, "_check_layout", lambda *a: (1, 2, 2, 2, 2, 128))
    monkeypatch.setattr(torch.cuda, "device", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(binding, "_new_workspace",
                        lambda like, n, stream: made.append((like is q, n, stream)) or torch.zeros(n, dtype=torch.uint8))
    assert binding.attn_fwd_splitkv_status(q, q, q, q, None, False, 1.0, 2, stream=0x1230) == 0
    assert made == [(True, 4096, 0x1230)] and calls[0][-2:] == (4096, 0x1230)
    own = torch.zeros(4096, dtype=torch.uint8)
    assert binding.attn_fwd_splitkv_status(q, q, q, q, None, False, 1.0, 2, workspace=own, stream=0x1230) == 0
    assert len(made) == 1 and calls[1][-3] == own.data_ptr()
