"""The stream that the binding passes where the caller names none."""
from types import SimpleNamespace

import pytest


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_without_torchs_private_handle_the_public_stream_serves(monkeypatch, missing):
    import torch

    import paper_2606_17421_amd as ck
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x10)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=0x20))
    assert ck._stream(None).value == 0x10
    monkeypatch.delattr(torch._C, missing)
    assert ck._stream(None).value == 0x20


@pytest.mark.gpu
def test_the_current_stream_is_passed(gpu_lib):
    import torch
    other = torch.cuda.Stream()
    for s in (torch.cuda.current_stream(), other):
        with torch.cuda.stream(s):
            assert (gpu_lib._stream(None).value or 0) == torch.cuda.current_stream().cuda_stream == s.cuda_stream
