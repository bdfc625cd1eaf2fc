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

    def tables(self, *a):
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


class FakeStream:
    cuda_stream = 77


@pytest.mark.parametrize("stream,at", [(None, 5), (FakeStream(), 77)])
def test_outputs_are_allocated_on_the_call_s_stream(host, stream, at):
    """Memory that the allocator hands out is free for the stream it was asked on: another's work may still read it."""
    from paper_2606_15157_gb300 import paged
    c = host
    c.fake.current = 5
    attend(c, stream=stream)  # (its scratch)
    del c.streams[:]
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    out = c.attention(q, None, None, stream=stream)
    assert [(s, t.data_ptr()) for s, t in c.streams] == [(at, out.data_ptr())] and out.shape == q.shape
    pool = object.__new__(paged.PagePool)
    pool._call, pool._lib, pool.free_count = (), c.fake, None
    del c.streams[:]
    lens = torch.zeros(2, dtype=torch.int32)
    got = pool.tables(lens, lens, 3, stream=stream)
    assert [s for s, _ in c.streams] == [at] * 5 and [t.data_ptr() for _, t in c.streams] == [t.data_ptr() for t in got]
    assert [t.numel() for t in got] == [2, 3, 3, 3, 2]
    del c.streams[:]
    pool.tables(lens, lens, 3, stream=stream, kv_lens=lens)  # some given
    assert [s for s, _ in c.streams] == [at] * 4


# ---- the extension module's calls, with a stub in the library's place ---------------------------------

@pytest.fixture(scope="module")
def stubbed(tmp_path_factory):
    """(module, stub): kvev_paged_bind linked against tests/paged_bind_stub.cpp."""
    import ctypes
    import importlib.util
    import os
    import subprocess

    from paper_2606_15157_gb300 import build
    build.build()
    tmp = tmp_path_factory.mktemp("bind")
    cflags, lflags = build._bind_flags()
    obj, so = str(tmp / "stub.o"), str(tmp / build.BIND)
    subprocess.run([build.CXX, *cflags, "-c", os.path.join(build.ROOT, "tests", "paged_bind_stub.cpp"), "-o", obj], check=True)
    subprocess.run([build.CXX, "-shared", "-Wl,-Bsymbolic", "-o", so, os.path.join(build.OBJDIR, "paged_bind.cpp.o"), obj,
                    *(f for f in lflags if "libkvev" not in f)], check=True)
    spec = importlib.util.spec_from_file_location("kvev_paged_bind", so)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m, ctypes.CDLL(so)


def on(device, dtype, *size):
    """A tensor that says it is on that GPU; nothing reads its memory."""
    stride = [1] * len(size)
    for i in range(len(size) - 2, -1, -1):
        stride[i] = stride[i + 1] * max(size[i + 1], 1)
    n = max(1, stride[0] * size[0]) * torch.empty(0, dtype=dtype).element_size()
    storage = torch._C._construct_storage_from_data_pointer(1 << 20, torch.device("cuda", device), n)
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        {"storage_offset": 0, "dtype": dtype, "size": size, "stride": tuple(stride)}, storage)


def bind_calls(m, dev):
    """The five calls on tensors of GPU `dev`, on a stream given by number."""
    import ctypes

    from paper_2606_15157_gb300 import kvev
    i32, bf = torch.int32, torch.bfloat16
    I = lambda *n: on(dev, i32, *n)  # noqa: E731
    global desc  # (the calls hold its address)
    desc = kvev.PagedCacheDesc(1 << 20, 1 << 20, 16 * 128, 128, 64, 8, 16, 2, 64, kvev.BF16)
    P = 1 << 20
    pool, cache = (16, 8, P, P, 2, 4, P, dev), (ctypes.addressof(desc), P, 2, 4, P, dev)
    rows, q, kv = on(dev, bf, 3, 2, 64), on(dev, bf, 3, 4, 64), on(dev, bf, 2, 2, 32, 64)
    return {"tables": lambda: m.tables(*pool, 5, I(2), I(2), 3, I(2), I(3), I(3), I(3), I(2), I(1), I(1)),
            "release": lambda: m.release(*pool, 5, I(2), I(2), I(2), I(1), I(1)),
            "write": lambda: m.write(*cache, 5, rows, rows, I(3)),
            "gather": lambda: m.gather(*cache, 5, I(2), kv, kv),
            "attention": lambda: m.attention(*cache, 5, q, I(3), I(2), q, None, 0.0, 0, P, 1 << 30)}


@pytest.mark.parametrize("name", ["tables", "release", "write", "gather", "attention"])
@pytest.mark.parametrize("current,dev", [(0, 1), (1, 0), (1, 1)])
def test_calls_run_on_the_tensors_gpu(stubbed, name, current, dev):
    import ctypes
    m, stub = stubbed
    at, seen = ctypes.c_int.in_dll(stub, "stub_device"), ctypes.c_int.in_dll(stub, "stub_seen")
    at.value, seen.value = current, -1
    assert bind_calls(m, dev)[name]() == 0
    assert seen.value == dev and at.value == current  # and the caller's device is current again


def test_a_refused_call_leaves_the_current_gpu(stubbed):
    import ctypes
    m, stub = stubbed
    at, calls = ctypes.c_int.in_dll(stub, "stub_device"), ctypes.c_int.in_dll(stub, "stub_calls")
    at.value = 0
    before = calls.value
    f = bind_calls(m, 1)
    wrong = on(0, torch.int32, 2)  # on another GPU than the cache
    with pytest.raises(ValueError):
        m.release(16, 8, 1 << 20, 1 << 20, 2, 4, 1 << 20, 1, 5, wrong, wrong, wrong, wrong, wrong)
    assert at.value == 0 and calls.value == before and f["write"]() == 0


# ---- sources ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("name", ["paged.cu", "paged_attn.cu", "paged.cuh"])
def test_overlapped_kernels_load_nothing_as_constant(name):
    """Launches that overlap the kernel before them read what it writes: no load may claim that it is constant while the grid exists."""
    import os
    import re

    from paper_2606_15157_gb300 import build
    with open(os.path.join(build.CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"__ldg\s*\(|\.global[.\w]*\.nc\b|__restrict__", code)


# ---- scratch given by the caller ------------------------------------------------------------------------

def test_scratch_given_is_checked_and_counted_in_bytes(host):
    c = host
    given = on(0, torch.float32, 1000)
    assert attend(c, workspace=given) == given.data_ptr() and c.fake.workspace_of_last()[1] == 4000
    made = len(c.fake.calls)
    rows = torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        {"storage_offset": 0, "dtype": torch.uint8, "size": (4, 8), "stride": (16, 1)}, given.untyped_storage())
    for bad in (torch.zeros(1000), on(1, torch.uint8, 1000), rows, 12345):
        with pytest.raises(ValueError):
            attend(c, workspace=bad)
    assert len(c.fake.calls) == made
