"""Where the decode-step operators' calls make their workspaces and results, on the host: the stream
that a raw handle stands for, with the device's own parts replaced by recorders."""
import contextlib

import pytest
import torch

from paper_2609_31395_amd import actkv


class FakeStream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index = handle, device_index


@pytest.fixture
def streams(monkeypatch):
    """torch.cuda with one device; `used` lists the streams that memory was made for."""
    used = []
    current = FakeStream(0x70)

    def external(handle, device=None):
        if not handle:   # what torch makes of a null handle: one of its own side streams
            return FakeStream(0x99)
        return FakeStream(handle)

    @contextlib.contextmanager
    def on(s):
        used.append(s.cuda_stream)
        yield
    monkeypatch.setattr(torch.cuda, "Stream", FakeStream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: FakeStream(0))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)   # a host tensor's device
    return used


@pytest.mark.parametrize("handle", [0, 0x70, 0x5000])
@pytest.mark.parametrize("raw", [True, False])
def test_memory_is_made_for_the_stream_of_the_call(streams, handle, raw):
    like = torch.zeros(4)
    with actkv._Launch(like, handle if raw else FakeStream(handle, -1)) as on:
        assert on.handle == handle
        on.scratch(64)
        on.result((3,), torch.float32)
    assert streams == [handle, handle]


@pytest.mark.parametrize("device", [0, 3])
def test_a_stream_of_another_device_is_refused(streams, device):
    with pytest.raises(ValueError, match="stream"):   # a host tensor's device is -1
        with actkv._Launch(torch.zeros(4), FakeStream(0x5000, device)):
            pass
    assert streams == []
