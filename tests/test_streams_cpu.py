"""Calls without a stream run on the current stream of the device that their tensors are on, whichever
device is the current one."""
import torch

from paper_2403_09636_amd import binding as Bd


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


def test_current_stream_of_the_tensors_device(monkeypatch):
    streams = {0: 4096, 1: 8192}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: streams[i], raising=False)
    for i, handle in streams.items():
        assert Bd._stream(None, torch.device("cuda", i)) == handle
    assert Bd._stream(_Stream(7), torch.device("cuda", 1)) == 7
    # torch without the raw handle
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: _Stream(streams[0 if dev is None else dev.index]))
    assert Bd._stream(None, torch.device("cuda", 1)) == 8192

