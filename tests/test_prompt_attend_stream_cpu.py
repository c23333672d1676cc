"""Where prompt_attend allocates its result, without a GPU: memory that a kernel writes on a
stream has to come from that stream's pool, or work of another stream may still use it."""
import contextlib

import pytest
import torch

from paper_2608_05326_amd import qevict as m


class Stream:
    device, cuda_stream = torch.device("cuda:0"), 5


@pytest.mark.parametrize("stream", [None, Stream()])
def test_the_result_comes_from_the_stream_that_writes_it(monkeypatch, stream):
    current, made, launched = ["main"], [], []

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    def rows(t, torch, index, name, *a):
        return t.data_ptr(), 0, 0

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: made.append(current[-1]) or empty(*a, **kw))
    monkeypatch.setattr(m, "_rows", rows)
    monkeypatch.setattr(m, "_int32", lambda *a: 0)
    monkeypatch.setattr(m, "_launch", lambda lib, torch, index, s, fn, *a: launched.append(s))
    q, k = torch.zeros(3, 4, 128), torch.zeros(3, 2, 128)
    cu = torch.tensor([0, 3], dtype=torch.int32)
    out = m.prompt_attend(q, k, k, cu, stream=stream)
    assert out.shape == q.shape and launched == [stream]
    assert made == ["main" if stream is None else stream]
    # a result of the caller's is its own business
    assert m.prompt_attend(q, k, k, cu, out, stream=stream) is out and len(made) == 1
