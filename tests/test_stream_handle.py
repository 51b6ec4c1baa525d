"""The stream a call goes to (no GPU needed: torch's answers are stood in for)."""
from types import SimpleNamespace

import torch

from paper_2404_14712_amd._lib import _stream


def test_given_streams():
    assert _stream(12) == 12 and _stream(SimpleNamespace(cuda_stream=34)) == 34


def test_current_stream_with_and_without_the_private_call(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=56))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert _stream(None) == 103
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert _stream(None) == 56
