"""The handle of the current stream that every entry point is given: with torch's quick way to it and without."""
import types

import pytest
import torch

from paper_2604_18780_amd import binding as sb


def test_without_the_quick_way(monkeypatch):
    monkeypatch.setattr(sb, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=1234))
    assert sb._stream() == 1234


@pytest.mark.gpu
def test_it_is_the_current_stream(monkeypatch):
    s = torch.cuda.Stream()
    for raw in (sb._raw_stream, None):
        monkeypatch.setattr(sb, "_raw_stream", raw)
        assert sb._stream() == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(s):
            assert sb._stream() == s.cuda_stream
