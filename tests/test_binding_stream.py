"""The stream that the binding hands to the library: the current one, by public names where torch has no others."""
import types

import pytest
import torch

from paper_2407_08103_amd import binding


def test_current_stream_by_public_names(monkeypatch):
    monkeypatch.setattr(binding, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert binding._stream(None) == 77


def test_current_stream_by_its_handle(monkeypatch):
    """torch.cuda.current_device() is asked, which makes torch ready for the GPU, or refuses where that cannot be."""
    asked = []
    monkeypatch.setattr(binding, "_raw_stream", lambda device: asked.append(device) or 88)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert binding._stream(None) == 88 and asked == [3]


def test_given_streams():
    assert binding._stream(5) == 5 and binding._stream(types.SimpleNamespace(cuda_stream=6)) == 6


@pytest.mark.gpu
def test_current_stream_on_the_gpu(monkeypatch):
    side = torch.cuda.Stream()
    for stream in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(stream):
            assert binding._stream(None) == stream.cuda_stream
            with monkeypatch.context() as m:
                m.setattr(binding, "_raw_stream", None)
                assert binding._stream(None) == stream.cuda_stream
