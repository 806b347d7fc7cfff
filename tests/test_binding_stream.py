"""The stream of a call that names none."""
import types

import torch

from paper_2607_24434_amd import _lib


def test_a_torch_without_the_raw_handle_gives_its_stream_object(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert _lib._stream(None) == 77


def test_the_raw_handle_is_of_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert _lib._stream(None) == 103
    assert _lib._stream(5) == 5
    assert _lib._stream(types.SimpleNamespace(cuda_stream=6)) == 6
