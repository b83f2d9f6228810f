"""The stream that a call without one works on: the current device's current one."""
import types

import torch

import paper_1812_08011_amd as fp8t


def test_current_stream(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert fp8t._stream(None) == 103
    # a torch that does not give the address alone
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert fp8t._stream(None) == 77


def test_given_streams():
    assert fp8t._stream(5) == 5
    assert fp8t._stream(types.SimpleNamespace(cuda_stream=6)) == 6
