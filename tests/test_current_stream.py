"""The current stream's handle as every entry point of the binding takes it, on any torch: by the short way where torch has it, by the
public one elsewhere (no GPU needed: torch's calls are replaced)."""
import types

import torch

from paper_2505_04421_amd import binding


def test_without_the_short_way(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=1234))
    assert binding._stream(None) == 1234


def test_the_short_way(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    assert binding._stream(None) == 1003
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    assert binding._stream(None) is None                      # the null stream


def test_streams_by_hand():
    assert binding._stream(77) == 77 and binding._stream(0) is None
    assert binding._stream(types.SimpleNamespace(cuda_stream=5)) == 5
