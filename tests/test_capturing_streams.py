"""On a host without a GPU: an object whose last call was on a stream that now
captures a graph.  An event recorded there would take the next stream, and the
call on it, into the graph, so the call is refused before one is."""
import os

import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.batch import StagingRing
from paper_2505_17074_amd.sample import Sampler


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


class _Stream:
    """Stands for a device's stream; `events` of its kind are recorded or waited for."""

    def __init__(self, handle):
        self.cuda_stream, self.events = handle, 0

    def record_event(self):
        self.events += 1

    def wait_event(self, event):
        self.events += 1


CAPTURING = {}


@pytest.fixture(autouse=True)
def streams(monkeypatch):
    CAPTURING.clear()
    monkeypatch.setattr(B, "stream_capturing", lambda h: CAPTURING.get(h, False))


def test_a_sampler():
    s, a, b = Sampler("cpu"), _Stream(1), _Stream(2)
    s._move(1, a)
    CAPTURING[1] = True
    with pytest.raises(RuntimeError, match="captur"):
        s._move(2, b)
    assert a.events == b.events == 0 and (s._last, s._last_h) == (a, 1)
    CAPTURING[1] = False
    s._move(2, b)
    assert a.events == b.events == 1 and (s._last, s._last_h) == (b, 2)


class _Event:
    def record(self, stream):
        stream.record_event()


def test_a_staging_ring(monkeypatch):
    monkeypatch.setattr(torch.cuda, "Event", _Event)
    r, a, b = StagingRing(), _Stream(1), _Stream(2)
    r._ring([None] * 4, 2)
    r._not_into_a_graph(a)
    r._order(a)
    r._done(r._slot(a), a)
    CAPTURING[1] = True
    with pytest.raises(RuntimeError, match="captur"):
        r._not_into_a_graph(b)
    assert a.events == b.events == 0 and r._last_stream is a and r._i == 1
    r._not_into_a_graph(a)
    CAPTURING[2] = True                        # both in one graph: it orders them
    r._not_into_a_graph(b)
    r._order(b)
    assert a.events == b.events == 1
    CAPTURING.clear()
    r._not_into_a_graph(a)


def test_a_verifier(monkeypatch):
    """Refused before it takes a slot, so that nothing is recorded for the slots
    used before either."""
    from paper_2505_17074_amd.batch import Verifier
    monkeypatch.setattr(torch.cuda, "Event", _Event)
    v, a, b = Verifier.__new__(Verifier), _Stream(1), _Stream(2)
    v._ring([None] * 4, 2)
    v._order(a)
    v._done(v._slot(a), a)
    CAPTURING[1] = True
    with pytest.raises(RuntimeError, match="captur"):
        v.run(stream=b)
    assert a.events == b.events == 0 and v._pending == [0]
