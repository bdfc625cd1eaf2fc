"""The host side of paged.py without a GPU: a fake of the extension module notes what each call hands to the library."""
import contextlib

import pytest
import torch


class FakeBind:
    """Streams by number; `capture` is the id of the capture that the stream is part of (0: none)."""

    def __init__(self):
        self.current, self.capture, self.calls = 0, 0, []

    def stream(self, device, stream):
        return (self.current if stream is None else stream), self.capture

    def attention(self, *a):
        self.calls.append(a)
        return 0

    def workspace_of_last(self):
        return self.calls[-1][-2:]


@pytest.fixture()
def host(monkeypatch):
    """(paged, cache): a PagedCache over the fake; new tensors are CPU tensors, their stream is noted in `streams`."""
    from paper_2606_15157_gb300 import build, kvev, paged
    build.build()
    kvev.load()
    fake = FakeBind()
    at = []
    real = torch.empty

    @contextlib.contextmanager
    def stream_context(s):
        at.append(getattr(s, "cuda_stream", s))
        yield
        at.pop()

    streams = []

    def empty(*a, **kw):
        kw.pop("device", None)
        t = real(*a, **kw)
        t.fill_(1)
        streams.append((at[-1] if at else fake.current, t))
        return t

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", stream_context)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda n, device=None: n)
    for name in ("_workspaces", "_captured"):
        monkeypatch.setattr(paged, name, {}, raising=False)
    monkeypatch.setattr(paged, "_bind", lambda: fake)
    c = object.__new__(paged.PagedCache)
    c._device, c._lib, c._call = 0, fake, (0, 0, 1, 1, 0, 0)
    c.fake, c.streams = fake, streams
    return c


def attend(c, **kw):
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    c.attention(q, None, None, out=q, **kw)
    return c.fake.workspace_of_last()[0]


def test_captures_have_scratch_of_their_own(host):
    c = host
    eager = attend(c)
    assert attend(c) == eager  # calls on a stream share it
    c.fake.capture = 7
    first = attend(c)
    assert attend(c) == first and c.workspace().data_ptr() == first
    c.fake.capture = 8  # the next graph on the same stream
    second = attend(c)
    assert len({eager, first, second}) == 3
    c.fake.capture = 0
    assert attend(c) == eager


def test_scratch_made_in_a_capture_is_not_taken_for_zeroed_outside(host):
    c = host
    c.fake.capture = 3  # the first call of all: its zeroing is a node of the graph
    captured = attend(c)
    c.fake.capture = 0
    eager = attend(c)
    assert eager != captured
    from paper_2606_15157_gb300 import kvev
    for _, t in c.streams:  # each has its counts zeroed where it was made
        assert not t[:kvev.PAGED_SYNC_BYTES].any()


def test_scratch_of_streams_forked_in_a_capture(host):
    c = host
    c.fake.capture = 3
    c.fake.current = 11
    a = attend(c)
    c.fake.current = 12
    b = attend(c)
    c.fake.current = 11
    assert a != b and attend(c) == a
