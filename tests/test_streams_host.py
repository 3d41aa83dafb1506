"""Which stream's memory the binding's own tensors come from, with torch's allocator and streams stood in for: a block that torch
keeps for the current stream may still be in use there when a call on another stream gets it."""
import contextlib

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld


class Stream:
    device_index, device = 0, torch.device("cuda", 0)

    def __init__(self, handle):
        self.cuda_stream = handle


class Block:
    """What torch.empty gives: it belongs to the stream that was current."""
    is_cuda = True

    def __init__(self, owner):
        self.owner, self.used_on = owner, []

    def record_stream(self, stream):
        if stream is not self.owner:  # torch passes over a block's own stream too
            self.used_on.append(stream)


@pytest.fixture
def streams(monkeypatch):
    main, side, third = Stream(0), Stream(16), Stream(32)
    current = [main]

    @contextlib.contextmanager
    def switched(stream):
        current.append(stream)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "stream", switched)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(ld, "_current_raw_stream", lambda index: current[-1].cuda_stream)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: Block(current[-1]))
    return main, side, third


def test_a_temporary_belongs_to_the_stream_that_uses_it(streams):
    main, side, third = streams
    t = ld._scratch(100, "cuda:0", None)
    assert t.owner is main and t.used_on == []
    t = ld._scratch(100, "cuda:0", main)
    assert t.owner is main and t.used_on == []
    t = ld._scratch(100, "cuda:0", side)
    assert t.owner is side and t.used_on == []


def test_a_temporary_of_two_streams(streams):
    main, side, third = streams
    for first, second in ((side, third), (side, None), (None, side), (side, side), (None, None)):
        t = ld._scratch(100, "cuda:0", first, second)
        assert t.owner is (first or main)
        assert t.used_on == [s for s in (second or main,) if s is not t.owner]


def test_an_output_belongs_to_the_stream_that_writes_it_and_may_be_read_on_the_current_one(streams):
    main, side, third = streams
    for stream in (None, main):
        t = ld._output(torch.float32, "cuda:0", stream, 3)
        assert t.owner is main and t.used_on == []
    t = ld._output(torch.float32, "cuda:0", side, 2, 3)
    assert t.owner is side and t.used_on == [main]


def test_host_memory_has_no_stream():
    assert ld._scratch(100, "cpu", Stream(16)).numel() == 100
    assert ld._output(torch.float32, torch.device("cpu"), Stream(16), 3).shape == (3,)
