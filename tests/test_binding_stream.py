"""The stream a call is put on: the caller's, or torch's current one."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def api():
    from paper_2606_03075_gb300 import api as _api
    return _api


@pytest.mark.parametrize("missing", ["_raw_stream", "_raw_device"])
def test_without_the_direct_accessors(api, monkeypatch, missing):
    """A torch without them: the public accessor gives the handle."""
    monkeypatch.setattr(api, missing, None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert api._stream(None) == 77
    assert api._stream(5) == 5


@pytest.mark.gpu
def test_both_ways_name_the_same_stream(api):
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            assert api._stream(None) == torch.cuda.current_stream().cuda_stream == stream.cuda_stream
    assert api._stream(side) == side.cuda_stream
