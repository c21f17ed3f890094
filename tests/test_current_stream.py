"""Which stream a call without one goes to: the current one, also where torch does not have the short way to ask for it.  No GPU is needed."""
from types import SimpleNamespace

import pytest


@pytest.mark.parametrize("short_way", [True, False])
def test_current_stream(monkeypatch, short_way):
    import torch
    import paper_2507_16274_amd as S
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: SimpleNamespace(cuda_stream=17))
    if short_way:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 17 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert S._stream(None) == 17
    assert S._stream(SimpleNamespace(cuda_stream=5)) == 5
