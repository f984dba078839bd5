"""The stream's handle as the binding takes it: torch's short way where there is one, its public one otherwise."""
import types

import torch

from paper_2509_26277_amd import binding


def test_public_way_without_the_short_one(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x1230))
    assert binding._stream() == 0x1230


def test_short_way_takes_the_current_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x4560 + device, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert binding._stream() == 0x4563
