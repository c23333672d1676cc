"""A stream of another device than the tensors' is refused before anything is enqueued (the
launch is not reached, so no GPU is needed)."""
import pytest
import torch

import paper_2608_05326_amd as qv
from paper_2608_05326_amd import qevict as m


class Stream:
    cuda_stream = 5

    def __init__(self, device):
        self.device = torch.device(device)


def test_calls_refuse_a_stream_of_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    called = []

    def fn(*a):
        called.append(a)
        return m.OK
    m._launch(None, torch, 0, Stream("cuda:0"), fn, 1)
    assert called == [(1, 5)]
    with pytest.raises(ValueError, match="cuda:1"):
        m._launch(None, torch, 0, Stream("cuda:1"), fn, 1)
    assert len(called) == 1


def test_a_cache_refuses_a_stream_of_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for device in ("cuda", "cuda:0"):
        with pytest.raises(ValueError, match="cuda:1"):
            qv.BlockCache(qv.BlockConfig(1, 2, 1, 64), device=device, stream=Stream("cuda:1"))
