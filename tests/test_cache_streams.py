"""The sampling and cache calls refuse a stream of another GPU than their tensors' before the library
sees it (no GPU needed)."""
import types

import pytest

from paper_2608_11235_amd import _lib, api


def test_a_stream_of_another_gpu(monkeypatch):
    called = []
    library = types.SimpleNamespace(cora_cache_plan=lambda *a: called.append(a) or 0)
    monkeypatch.setattr(_lib, "load", lambda: library)
    monkeypatch.setattr(api.torch.cuda, "current_device", lambda: 0)
    stream = types.SimpleNamespace(device_index=1, cuda_stream=99)
    with pytest.raises(ValueError, match="stream: on cuda:1"):
        api._call(0, "cora_cache_plan", 1, 2, stream=stream)
    assert not called
    stream.device_index = 0
    api._call(0, "cora_cache_plan", 1, 2, stream=stream)
    assert called == [(1, 2, 99)]
