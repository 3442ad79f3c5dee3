"""Which stream a chunk plan's memory is taken to come from when its cache lies on another GPU than the current one."""
import types

import pytest
import torch

from paper_2609_19242_amd import chunk as km


@pytest.mark.parametrize("stream,want", [(None, {77}), (55, {55})])
def test_the_stream_of_the_plans_own_gpu(monkeypatch, stream, want):
    # (111: the current stream of the current GPU, which must not be recorded for tensors of GPU 1)
    monkeypatch.setattr(km, "_stream", lambda s: 111 if s is None else s)
    monkeypatch.setattr(km, "_raw_stream", lambda device: {1: 77}[device], raising=False)
    cache = types.SimpleNamespace(dtype=torch.bfloat16, device=torch.device("cuda", 1), gpu=1, head_dim=64)
    plan = km.ChunkPlan(cache, km._Chunk(2, 6, 1, 0, 4, 0, 0.0, 0), torch.zeros(64, dtype=torch.int32), stream)
    assert plan._streams == want
