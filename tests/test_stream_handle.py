"""The handle of the current stream, by torch's own interface where a torch has no shorter way; no GPU needed."""
import types

import torch

from paper_2510_23938_b200 import binding


def test_without_the_short_way(monkeypatch):
    monkeypatch.setattr(binding, "_current_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=77))
    assert binding._stream_ptr(None) == 77
    assert binding._stream_ptr(types.SimpleNamespace(cuda_stream=5)) == 5


def test_the_short_way_is_that_of_the_current_device(monkeypatch):
    asked = []
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: asked.append(device) or 99)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert binding._stream_ptr(None) == 99 and asked == [3]
    assert binding._stream_ptr(types.SimpleNamespace(cuda_stream=5)) == 5 and asked == [3]
