"""Which stream a call without one goes to: torch's current stream of the current device."""
import types

import pytest
import torch

from paper_2506_03781_amd import uniquan as uq

RAW = "_cuda_getCurrentRawStream"


def test_without_torchs_private_call(monkeypatch):
    """The handle's short way is private to torch; where it is missing the public one serves."""
    monkeypatch.delattr(torch._C, RAW, raising=False)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert uq._stream(None) == 77


def test_current_device_and_given_streams(monkeypatch):
    monkeypatch.setattr(torch._C, RAW, lambda device: 100 + device, raising=False)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    assert uq._stream(None) == 103
    assert uq._stream(types.SimpleNamespace(cuda_stream=5)) == 5
    assert uq._stream(6) == 6 and uq._stream(0) == 0


@pytest.mark.gpu
def test_both_ways_agree(monkeypatch):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    side = torch.cuda.Stream()
    for st in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(st):
            assert uq._stream(None) == st.cuda_stream
            with monkeypatch.context() as m:
                m.delattr(torch._C, RAW)
                assert uq._stream(None) == st.cuda_stream
            g = torch.cuda.CUDAGraph()
            x = torch.zeros(4, device="cuda")
            torch.cuda.synchronize()
            if st is side:
                with torch.cuda.graph(g, stream=side):
                    assert uq._stream(None) == side.cuda_stream
                    x += 1
                g.replay()
    torch.cuda.synchronize()
