"""Which stream a call without one runs on."""
from types import SimpleNamespace

import pytest
import torch

from paper_1707_02402_amd import binding


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_a_torch_without_the_short_way_is_asked_for_its_current_stream(monkeypatch, missing):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x50 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=0x1230))
    assert binding._stream().value == 0x53
    monkeypatch.delattr(torch._C, missing)
    assert binding._stream().value == 0x1230
    assert binding._stream(SimpleNamespace(cuda_stream=0x77)).value == 0x77


@pytest.mark.gpu
def test_both_ways_name_the_same_stream():
    assert torch.cuda.is_available()
    handle = lambda: (binding._stream().value or 0, torch.cuda.current_stream().cuda_stream)
    first = handle()
    assert first[0] == first[1]
    with torch.cuda.stream(torch.cuda.Stream()):
        inside = handle()
        assert inside[0] == inside[1] != first[0]
    assert handle() == first
