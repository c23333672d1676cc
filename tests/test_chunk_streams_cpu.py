"""On which stream a chunk step's own tensor work is enqueued, and where the rotation allocates its
results, without a GPU (as in the models of test_block_cache_streams_cpu.py and
test_prompt_attend_stream_cpu.py)."""
import contextlib

import pytest
import torch

from paper_2608_05326_amd import qevict as m
from test_block_cache_streams_cpu import machine  # noqa: F401  (a fixture)


def _cu(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_advance_and_the_calls_follow_the_stream_of_the_cache(machine, monkeypatch):  # noqa: F811
    cache = m.BlockCache(m.BlockConfig(3, 8, 2, 200, chunk_tokens=16), stream=machine.side)
    cache.lens = _cu(0, 100, -1)
    cu, counts = _cu(0, 5, 9, 9), _cu(2, 4, 0)
    q, k = torch.zeros(9, 8, 128, dtype=torch.bfloat16), torch.zeros(9, 2, 128, dtype=torch.bfloat16)
    machine.take()
    launched = []
    monkeypatch.setattr(m, "_launch", lambda lib, t, index, stream, fn, *a: launched.append(stream))
    monkeypatch.setattr(m, "_rows", lambda t, *a: (0, 0, 0))
    monkeypatch.setattr(m, "_int32", lambda *a: 0)
    cache.attend_chunk(0, q, k, k, cu, q)
    cache.append(0, k, k, cu, counts=counts)
    assert launched == [machine.side] * 2 and not machine.take()
    cache.advance(cu, counts)
    log = machine.take()
    assert log and {x[0] for x in log} == {"side"}
    assert cache.lens.tolist() == [2, 104, -1]


class Stream:
    device, cuda_stream = torch.device("cuda:0"), 5


@pytest.mark.parametrize("stream", [None, Stream()])
def test_rotated_rows_come_from_the_stream_that_writes_them(monkeypatch, stream):
    current, made, launched = ["main"], [], []

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    new_empty = torch.Tensor.new_empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda x, *a: made.append(current[-1]) or new_empty(x, *a))
    monkeypatch.setattr(m, "_rows", lambda t, *a: (t.data_ptr(), 0, 0))
    monkeypatch.setattr(m.Rotary, "_positions", lambda *a: (0, 0, 0))
    monkeypatch.setattr(m, "_launch", lambda lib, t, index, s, fn, *a: launched.append(s))
    q, k, r = torch.zeros(3, 4, 128), torch.zeros(3, 2, 128), m.Rotary()
    qo, ko = m.rotate(q, k, None, r, stream=stream)
    assert qo.shape == q.shape and ko.shape == k.shape and launched == [stream]
    assert made == ["main" if stream is None else stream] * 2
    qo, none = m.rotate(q, None, None, r, stream=stream)
    assert none is None and len(made) == 3
    # results of the caller's are its own business
    qo, ko = m.rotate(q, k, None, r, q_out=q, k_out=k, stream=stream)
    assert qo is q and ko is k and len(made) == 3
