"""The bindings' default stream, with and without torch's shortcut to its handle."""
from types import SimpleNamespace

import torch

from paper_2512_13282_gb300 import gemm as G


def test_default_stream_without_the_private_shortcut(monkeypatch):
    """torch._C._cuda_getCurrentRawStream is no public function: a torch
    without it gives the handle by its stream object."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: SimpleNamespace(cuda_stream=0x77))
    assert G._stream(None) == 0x77


def test_default_stream_is_that_of_the_current_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x50 + device, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert G._stream(None) == 0x53


def test_given_streams():
    assert G._stream(0) == 0 and G._stream(SimpleNamespace(cuda_stream=9)) == 9
