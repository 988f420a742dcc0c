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
