"""The stream that a call without one goes to, on the CPU: stand-ins for torch's."""
import types

import pytest
import torch

from paper_2506_24119_amd import binding as sb


def test_given_streams_pass_through():
    assert sb._stream_handle(77) == 77 and sb._stream_handle(types.SimpleNamespace(cuda_stream=5)) == 5


@pytest.mark.parametrize("private", [True, False])
def test_the_current_stream_with_and_without_the_private_call(monkeypatch, private):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=1234))
    if private:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 1000 + d, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert sb._stream_handle(None) == (1003 if private else 1234)
