"""The stream that calls go to, with and without torch's short way to its handle."""
import types

import pytest
import torch

from paper_2510_03425_amd import device as D


def test_a_torch_without_the_short_way(monkeypatch):
    monkeypatch.setattr(D, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert D.stream_handle() == 77


@pytest.mark.gpu
def test_both_ways_give_the_current_stream(gpu, monkeypatch):
    side = torch.cuda.Stream()
    for s in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(s):
            short = D.stream_handle()
            with monkeypatch.context() as m:
                m.setattr(D, "_raw_stream", None)
                assert D.stream_handle() == short == s.cuda_stream
