"""On which stream the binding's own tensor work is enqueued, without a GPU: the device calls
are replaced by a model of streams (a current one, waits between them) and every torch
operation is noted with the stream that is current when it runs."""
import contextlib

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import paper_2608_05326_amd as qv


class Stream:
    def __init__(self, name, log, device="cuda:0"):
        self.name, self.log, self.device, self.cuda_stream = name, log, torch.device(device), 0

    def wait_stream(self, other):
        self.log.append((self.name, "wait", other.name))


class Noted(TorchDispatchMode):
    def __init__(self, machine):
        super().__init__()
        self.machine = machine

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if func.overloadpacket.__name__ != "select":   # a view: nothing is enqueued
            self.machine.log.append((self.machine.current.name, func.overloadpacket.__name__, None))
        return func(*args, **(kwargs or {}))


class Machine:
    def __init__(self):
        self.log = []
        self.main, self.side = Stream("main", self.log), Stream("side", self.log)
        self.current = self.main

    @contextlib.contextmanager
    def on(self, stream):
        before, self.current = self.current, stream
        try:
            yield
        finally:
            self.current = before

    def take(self):
        log, self.log[:] = list(self.log), []
        return log


@pytest.fixture
def machine(monkeypatch):
    m = Machine()
    for name in ("zeros", "full", "empty"):
        make = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, make=make, device=None, **kw: make(*a, **kw))
    monkeypatch.setattr(torch.cuda, "stream", m.on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: m.current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with Noted(m):
        yield m


def _cache(machine, num_pages, stream):
    c = qv.BlockCache(qv.BlockConfig(3, 8, 2, 200, num_pages=num_pages), stream=stream)
    return c, machine.take()


@pytest.mark.parametrize("num_pages", [0, 7])
def test_a_cache_with_a_stream_is_filled_on_it(machine, num_pages):
    _, log = _cache(machine, num_pages, machine.side)
    ops = [x for x in log if x[1] != "wait"]
    assert len(ops) >= 9 and {x[0] for x in ops} == {"side"}
    # what the creating stream does with the tensors comes after the fills
    assert log[-1] == ("main", "wait", "side")


def test_advance_follows_the_steps_of_the_cache(machine):
    cache, _ = _cache(machine, 0, machine.side)
    cache.advance()
    log = machine.take()
    assert log and {x[0] for x in log} == {"side"}


@pytest.mark.parametrize("name", ["lens", "table"])
def test_an_assigned_value_is_copied_between_two_waits(machine, name):
    """After the work that makes the value, behind the cache's pending calls, and before the
    program's stream may change the value again."""
    cache, _ = _cache(machine, 0, machine.side)
    value = torch.ones_like(getattr(cache, name))
    machine.take()
    setattr(cache, name, value)
    log = machine.take()
    assert log[0] == ("side", "wait", "main") and log[-1] == ("main", "wait", "side")
    assert len(log) > 2 and {x[0] for x in log[1:-1]} == {"side"}
    assert bool((getattr(cache, name) == 1).all())


def test_nothing_waits_where_there_is_one_stream(machine):
    cache, log = _cache(machine, 0, None)
    cache.lens = torch.zeros(3, dtype=torch.int32)
    cache.advance()
    assert not [x for x in log + machine.take() if x[1] == "wait" or x[0] != "main"]
    assert cache.lens.tolist() == [1, 1, 1]
    with machine.on(machine.side):
        cache, _ = _cache(machine, 0, machine.side)
        cache.lens = torch.zeros(3, dtype=torch.int32)
        cache.advance()
        assert not [x for x in machine.take() if x[1] == "wait" or x[0] != "side"]
