"""Calls with a stream of their own run on the current device too: tensors of another one are refused (no GPU needed)."""
import types

import pytest
import torch

from paper_2608_03447_gb300 import asd

ON_1 = types.SimpleNamespace(cuda_stream=0x5eed, device=torch.device("cuda", 1))


@pytest.mark.parametrize("stream", (None, ON_1, types.SimpleNamespace(cuda_stream=0x5eed), 0x5eed),
                         ids=("none", "torch", "no device", "handle"))
def test_another_current_device(monkeypatch, stream):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="on cuda:1, the current device is cuda:0"):
        asd._stream_at(stream, 1)


def test_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(asd, "_raw_stream", lambda device: 0x100 + device)
    assert asd._stream_at(None, 1) == 0x101
    assert asd._stream_at(ON_1, 1) == asd._stream_at(0x5eed, 1) == 0x5eed
    with pytest.raises(ValueError, match="its stream is on cuda:2"):
        asd._stream_at(types.SimpleNamespace(cuda_stream=1, device=torch.device("cuda", 2)), 1)
