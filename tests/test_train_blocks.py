"""Memory of quantised matrices that other streams read: noting the readers, and giving it back once they
are waited for.  On the CPU, with streams and an allocator that only keep books."""
import itertools
import sys
import threading
import time

import pytest

from paper_2603_18112_gb300 import mx


class Streams:
    """Streams by their handles, 0 the default one: which are under capture, who waited for whom, what
    was given back."""

    def __init__(self):
        self.here = threading.local()
        self.capturing, self.waits, self.freed, self.on_wait = set(), [], [], None
        self.addresses = itertools.count(0x1000, 0x1000)

    @property
    def current(self):
        return getattr(self.here, "stream", 0)

    def handle(self, stream):
        outer = self

        class Stream:
            cuda_stream = stream

            def wait_stream(self, other):
                outer.waits.append((stream, other.cuda_stream))
                if outer.on_wait:
                    outer.on_wait(stream, other.cuda_stream)

        return Stream()

    def on(self, stream):
        outer = self

        class On:
            def __enter__(self):
                self.before, outer.here.stream = outer.current, stream.cuda_stream

            def __exit__(self, *_):
                outer.here.stream = self.before

        return On()

    def alloc(self, size, stream):
        return next(self.addresses)

    def block(self, stream, readers=()):
        """One made on `stream` and read on `readers`."""
        with self.on(self.handle(stream)):
            block = mx._Block(256, 0, self.alloc)
        for r in readers:
            self.read(block, r)
        return block

    def read(self, block, stream):
        with self.on(self.handle(int(stream))):
            block.read_elsewhere(stream)


@pytest.fixture
def streams(monkeypatch):
    s = Streams()

    class Device:
        def __init__(self, _):
            pass

        def __enter__(self):
            pass

        def __exit__(self, *_):
            pass

    monkeypatch.setattr(mx, "_raw_stream", lambda device: s.current)
    monkeypatch.setattr(mx, "_get_device", lambda: 0)
    monkeypatch.setattr(mx, "_unfreed", [])
    monkeypatch.setattr(mx._Block.__del__, "__defaults__", (s.freed.append,))
    monkeypatch.setattr(mx, "_raw_delete", s.freed.append, raising=False)
    monkeypatch.setattr(mx.torch.cuda, "device", Device)
    monkeypatch.setattr(mx.torch.cuda, "stream", s.on)
    monkeypatch.setattr(mx.torch.cuda, "ExternalStream", lambda handle, device: s.handle(handle))
    monkeypatch.setattr(mx.torch.cuda, "default_stream", lambda device: s.handle(0))
    monkeypatch.setattr(mx.torch.cuda, "is_current_stream_capturing", lambda: s.current in s.capturing)
    return s


def test_readers_are_waited_for(streams):
    block = streams.block(7, [8, 9, 8])
    ptr = block.ptr
    del block
    assert sorted(streams.waits) == [(7, 8), (7, 9)] and streams.freed == [ptr]
    block = streams.block(7)
    ptr = block.ptr
    del block
    assert len(streams.waits) == 2 and streams.freed[1:] == [ptr]


def test_readers_noted_at_the_same_time_are_all_kept(streams):
    """A thread notes its stream in the middle of another thread's note."""
    block = streams.block(7)

    class Slow(int):
        between = None

        def __hash__(self):
            if Slow.between:
                between, Slow.between = Slow.between, None
                between()
            return int.__hash__(self)

    Slow.between = lambda: streams.read(block, 9)
    streams.read(block, Slow(8))
    assert block.readers == {8, 9}


def test_a_reader_that_is_noted_costs_no_more(streams, monkeypatch):
    """Weights that are read on one stream again and again: from the second time on nothing is asked."""
    block = streams.block(7, [8])

    def none(*_):
        raise AssertionError

    with monkeypatch.context() as m:
        m.setattr(mx.torch.cuda, "device", none)
        m.setattr(mx.torch.cuda, "is_current_stream_capturing", none)
        streams.read(block, 8)
    assert block.readers == {8}


def _held(streams, blocks):
    """Drops blocks while their streams are under capture, so that they wait for a later call."""
    ptrs = [b.ptr for b in blocks]
    streams.capturing |= {b.stream for b in blocks}
    blocks.clear()
    assert not streams.freed and len(mx._unfreed) == len(ptrs)
    streams.capturing.clear()
    return ptrs


def test_each_block_is_given_back_once(streams):
    """Two give blocks back at the same time: one begins in the middle of the other's waits, as another
    thread's or the collector's may."""
    blocks = [streams.block(7, [8]), streams.block(7, [9]), streams.block(6, [8])]
    ptrs = _held(streams, blocks)

    def again(*_):
        streams.on_wait = None
        mx._free_after_readers(streams.freed.append)

    streams.on_wait = again
    mx._free_after_readers(streams.freed.append)
    assert sorted(streams.freed) == ptrs and not mx._unfreed


def test_each_block_is_given_back_once_by_threads(streams):
    errors = []

    def hook(unraisable):
        errors.append(unraisable)

    before, sys.unraisablehook = sys.unraisablehook, hook
    streams.on_wait = lambda *_: time.sleep(1e-5)
    ptrs = []

    def drop(stream):
        for _ in range(200):
            block = streams.block(stream, [8, 9])
            ptrs.append(block.ptr)
            del block

    try:
        threads = [threading.Thread(target=drop, args=(s,)) for s in (4, 5, 6, 7)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        mx._free_after_readers(streams.freed.append)
    finally:
        sys.unraisablehook = before
    assert not errors and not mx._unfreed
    assert len(streams.freed) == 800 and sorted(streams.freed) == sorted(ptrs)


def test_a_stream_that_cannot_be_waited_for(streams):
    """Its block stays where it is, and the others are given back."""
    blocks = [streams.block(7, [8]), streams.block(7, [9]), streams.block(6, [8])]
    ptrs = _held(streams, blocks)

    def gone(own, reader):
        if reader == 9:
            raise RuntimeError("no such stream")

    streams.on_wait = gone
    mx._free_after_readers(streams.freed.append)
    assert sorted(streams.freed) == [ptrs[0], ptrs[2]] and not mx._unfreed


def test_a_block_dropped_under_capture_goes_back_after_it(streams):
    """With the next block that is made, also where no other one is ever read elsewhere; not while the
    stream that one is made on is under capture itself."""
    block = streams.block(7, [8])
    ptr = block.ptr
    streams.capturing.add(8)
    del block
    streams.block(6)
    assert ptr not in streams.freed
    streams.capturing.add(6)
    streams.capturing.remove(8)
    streams.block(6)
    assert ptr not in streams.freed and not streams.waits
    streams.capturing.clear()
    streams.block(6)
    assert ptr in streams.freed and streams.waits == [(7, 8)] and not mx._unfreed


def test_a_block_made_under_capture_is_not_handed_out_within_it(streams):
    """Read on a second stream of the capture: its memory would go to the capture's next block, which the
    graph may fill while the reader's branch still runs.  A block from before the capture is the caller's
    to keep, and no reader is noted."""
    before = streams.block(5)
    streams.capturing |= {7, 8}
    block = streams.block(7, [8])
    ptr = block.ptr
    assert block.readers == {8}
    streams.read(before, 8)
    streams.read(before, 7)
    assert before.readers is None
    del block
    streams.block(7)
    assert ptr not in streams.freed
    streams.capturing.clear()
    streams.block(6)
    assert ptr in streams.freed and not mx._unfreed
