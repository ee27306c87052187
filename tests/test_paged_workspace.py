"""Whose a PagedCache's workspace is, without a GPU: torch's allocator and streams are stand-ins that keep a list of what is asked of them."""
import contextlib
import types

import pytest
import torch

from paper_2503_01330_amd import binding as wkv
from test_paged_boundary import P, cache


class Stream:
    def __init__(self, address, device=None):
        self.cuda_stream = address

    def synchronize(self):
        Stream.log.append(("wait", self.cuda_stream))


class Memory:
    def __init__(self, size):
        self.size = size

    numel = lambda self: self.size                           # noqa: E731
    data_ptr = lambda self: P                                # noqa: E731

    def record_stream(self, stream):
        Stream.log.append(("used", self, stream.cuda_stream))


@pytest.fixture
def made(monkeypatch):
    """A PagedCache whose calls go nowhere; .now: the current stream, .capturing: streams that record a graph."""
    now = types.SimpleNamespace(stream=7, capturing=set(), taken=[])
    Stream.log = []

    def empty(size, **kw):
        now.taken.append(Memory(size))
        Stream.log.append(("taken", now.stream))
        return now.taken[-1]

    @contextlib.contextmanager
    def on(s):
        before, now.stream = now.stream, s.cuda_stream
        yield
        now.stream = before

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(now.stream))
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now.stream in now.capturing)
    monkeypatch.setattr(wkv, "_current_stream", lambda: now.stream)
    monkeypatch.setattr(wkv, "_current_device", lambda: 0)
    monkeypatch.setattr(wkv, "_paged_step", lambda *a: Stream.log.append(("step", a[-1])) or 0)
    c = wkv.PagedCache.__new__(wkv.PagedCache)
    c.c, c.batch, c.index, c.device, c._kept, c._work, c._streams = cache(score_stride=128), 3, 0, "cuda:0", [], None, set()
    c._ref = c._rows_ref = 0
    c._fill = lambda *a: None
    c.now = now
    return c


def test_memory_taken_anew_is_waited_for(made):
    """On the stream that it is taken on, before any call may have it."""
    made._reserve(0, 0)
    assert Stream.log == [("taken", 7), ("wait", 7)]
    made._reserve(0, 0)
    assert len(Stream.log) == 2                             # (there already)


def test_memory_waits_for_every_stream_that_it_was_used_on(made):
    made._reserve(0, 0)
    del Stream.log[:]
    work = made.now.taken[0]
    made.step(None, None, None, None)
    made.step(None, None, None, None, stream=9)
    made.step(None, None, None, None, stream=9)
    made.now.stream = 0
    made.step(None, None, None, None)
    assert Stream.log == [("step", 7), ("used", work, 9), ("step", 9), ("step", 9), ("used", work, 0), ("step", 0)]
    del Stream.log[:]
    made._reserve(100000, 1000, 9)                           # another, taken on stream 0
    made.step(None, None, None, None, stream=9)
    assert Stream.log == [("taken", 0), ("wait", 0), ("used", made.now.taken[1], 9), ("step", 9)] and work in made._kept


@pytest.mark.parametrize("current,stream", [(7, None), (7, 7), (7, 9), (9, 7)])
def test_no_memory_is_taken_while_a_graph_is_recorded(made, current, stream):
    made.now.capturing, made.now.stream = {9 if 9 in (current, stream) else 7}, current
    with pytest.raises(wkv.WkvError, match="recorded"):
        made._reserve(0, 0, stream)
    assert not made.now.taken and made._work is None
