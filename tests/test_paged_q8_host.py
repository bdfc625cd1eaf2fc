"""The host side of the 8-bit caches and of shared prefixes without a GPU: what each call hands to the library, and on which GPU."""
import ctypes
import os
import re

import pytest
import torch

from tests.test_paged_host import FakeStream, host, on  # noqa: F401


class FakeQ8:
    def __init__(self):
        self.calls = []

    def attention(self, *a):
        self.calls.append(a)
        return 0

    attention_shared = attention


@pytest.fixture()
def q8(host, monkeypatch):  # noqa: F811
    """(16-bit cache, 8-bit cache, fake of the q8 calls) over the fakes."""
    from paper_2606_15157_gb300 import paged
    fake = FakeQ8()
    monkeypatch.setattr(paged, "_bind_q8", lambda: fake)
    host.H_kv, host.d = 1, 64
    c = object.__new__(paged.QuantizedCache)
    c._device, c._lib, c._q8, c._call = 0, host.fake, fake, (0, 0, 1, 1, 0, 0)
    return host, c, fake


def shared(c, T, fake, **kw):
    q = torch.zeros((T, 1, 64), dtype=torch.bfloat16)
    c.attention_shared(q, None, None, None, None, out=q, **kw)
    return fake.calls[-1][-2:]


def test_the_scratch_of_a_stream_grows_and_is_shared(q8):
    from paper_2606_15157_gb300 import kvev, paged
    c, q, fake = q8
    a = shared(c, 10, fake)
    assert a[1] >= kvev.kvev_paged_attention_shared_workspace(1, 1, 64, 10)
    assert shared(c, 8, fake) == a  # large enough
    b = shared(c, 100000, fake)
    assert b != a and b[1] >= kvev.kvev_paged_attention_shared_workspace(1, 1, 64, 100000)
    assert shared(c, 10, fake) == b
    assert (c.workspace().data_ptr(), c.workspace().numel()) == b
    t = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    q.attention(t, None, None, out=t)  # every layer's calls on the stream take it
    assert fake.calls[-1][-2:] == b
    for _, s in c.streams:
        assert not s[:kvev.PAGED_SYNC_BYTES].any()
    assert len(paged._workspaces) == 1


def test_captures_grow_scratch_of_their_own(q8):
    c, q, fake = q8
    eager = shared(c, 10, fake)
    c.fake.capture = 7
    a = shared(c, 10, fake)
    b = shared(c, 100000, fake)
    assert len({eager[0], a[0], b[0]}) == 3 and shared(c, 10, fake) == b
    c.fake.capture = 0
    assert shared(c, 10, fake) == eager


@pytest.mark.parametrize("stream,at", [(None, 5), (FakeStream(), 77)])
def test_outputs_are_allocated_on_the_call_s_stream(q8, stream, at):
    c, q, fake = q8
    c.fake.current = 5
    x = torch.zeros((3, 1, 64), dtype=torch.bfloat16)
    for f in (lambda: c.attention_shared(x, None, None, None, None, stream=stream), lambda: q.attention(x, None, None, stream=stream)):
        f()  # (the scratch)
        del c.streams[:]
        out = f()
        assert [(s, t.data_ptr()) for s, t in c.streams] == [(at, out.data_ptr())] and out.shape == x.shape


# ---- the extension module's calls, with a stub in the library's place ---------------------------------

@pytest.fixture(scope="module")
def stubbed(tmp_path_factory):
    import importlib.util
    import subprocess

    from paper_2606_15157_gb300 import build
    build.build()
    tmp = tmp_path_factory.mktemp("bind")
    cflags, lflags = build._bind_flags()
    obj, so = str(tmp / "stub.o"), str(tmp / "kvev_paged_q8_bind.so")
    subprocess.run([build.CXX, *cflags, "-c", os.path.join(build.ROOT, "tests", "paged_q8_bind_stub.cpp"), "-o", obj], check=True)
    subprocess.run([build.CXX, "-shared", "-Wl,-Bsymbolic", "-o", so, os.path.join(build.OBJDIR, "paged_q8_bind.cpp.o"), obj,
                    *(f for f in lflags if "libkvev" not in f)], check=True)
    spec = importlib.util.spec_from_file_location("kvev_paged_q8_bind", so)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m, ctypes.CDLL(so)


def bind_calls(m, dev):
    from paper_2606_15157_gb300 import kvev
    i32, bf = torch.int32, torch.bfloat16
    I = lambda *n: on(dev, i32, *n)  # noqa: E731
    P = 1 << 20
    global held  # (the calls hold their addresses)
    held = (kvev.PagedQ8CacheDesc(P, P, P, P, 16 * 128, 128, 64, 32, 8, 16, 2, 64, kvev.BF16),
            kvev.PagedCacheDesc(P, P, 16 * 128, 128, 64, 8, 16, 2, 64, kvev.BF16))
    c8, c16 = ((ctypes.addressof(d), P, 2, 4, P, dev) for d in held)
    rows, q, kv = on(dev, bf, 3, 2, 64), on(dev, bf, 3, 4, 64), on(dev, bf, 2, 2, 32, 64)
    return {"write": lambda: m.write(*c8, 5, rows, rows, I(3)), "gather": lambda: m.gather(*c8, 5, I(2), kv, kv),
            "attention": lambda: m.attention(*c8, 5, q, I(3), I(2), q, None, 0.0, 0, P, 1 << 30),
            "attention_shared": lambda: m.attention_shared(*c16, 5, q, I(3), I(2), I(2), I(1), q, None, 0.0, P, 1 << 30)}


@pytest.mark.parametrize("name", ["write", "gather", "attention", "attention_shared"])
@pytest.mark.parametrize("current,dev", [(0, 1), (1, 0), (1, 1)])
def test_calls_run_on_the_tensors_gpu(stubbed, name, current, dev):
    m, stub = stubbed
    at, seen = ctypes.c_int.in_dll(stub, "stub_device"), ctypes.c_int.in_dll(stub, "stub_seen")
    at.value, seen.value = current, -1
    assert bind_calls(m, dev)[name]() == 0
    assert seen.value == dev and at.value == current  # and the caller's device is current again


def test_a_refused_call_reaches_nothing(stubbed):
    m, stub = stubbed
    at, calls = ctypes.c_int.in_dll(stub, "stub_device"), ctypes.c_int.in_dll(stub, "stub_calls")
    at.value = 0
    bind_calls(m, 1)
    before = calls.value
    P, I = 1 << 20, lambda dev, *n: on(dev, torch.int32, *n)  # noqa: E731
    q = on(1, torch.bfloat16, 3, 4, 64)
    c16 = (ctypes.addressof(held[1]), P, 2, 4, P, 1, 5)
    for groups, lens in ((I(0, 2), I(1, 1)), (I(1, 3), I(1, 1)), (I(1, 2), on(1, torch.float32, 1)), (None, I(1, 1))):
        with pytest.raises(ValueError):
            m.attention_shared(*c16, q, I(1, 3), I(1, 2), groups, lens, q, None, 0.0, P, 1 << 30)
    with pytest.raises(TypeError):
        m.attention_shared(*c16, q)
    assert at.value == 0 and calls.value == before


@pytest.mark.parametrize("name", ["paged_attn.cuh", "paged_shared.cu", "paged_q8.cu", "paged_q8_attn.cu", "paged_q8_few.cuh"])
def test_overlapped_kernels_load_nothing_as_constant(name):
    """Launches that overlap the kernel before them read what it writes: no load may claim that it is constant while the grid exists."""
    from paper_2606_15157_gb300 import build
    with open(os.path.join(build.CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"__ldg\s*\(|\.global[.\w]*\.nc\b|__restrict__", code)


@pytest.mark.parametrize("call", ["attention", "shared", "q8"])
@pytest.mark.parametrize("capture", [0, 7])
def test_scratch_outlives_the_launch_that_it_was_looked_up_for(q8, call, capture, monkeypatch):
    """Between one thread's look-up and its launch another's call on the stream may put a larger scratch in its place."""
    import gc
    import weakref

    from paper_2606_15157_gb300 import paged
    c, q, fake = q8
    c.fake.capture = capture
    x = torch.zeros((3, 1, 64), dtype=torch.bfloat16)
    calls = {"attention": lambda: c.attention(x, None, None, out=x), "q8": lambda: q.attention(x, None, None, out=x),
             "shared": lambda: c.attention_shared(x, None, None, None, None, out=x)}
    calls[call]()  # (the stream's scratch)
    tensors = [weakref.ref(t) for _, t in c.streams if t.dtype is torch.uint8]
    del c.streams[:]
    alive, inside = [], []

    def launched(*a):
        if not inside:
            inside.append(a[-2])
            shared(c, 100000, fake)  # the other thread's
            del c.streams[:]
            gc.collect()
            alive.extend(t().data_ptr() for t in tensors if t() is not None)
        return fake_calls(*a)

    def fake_calls(*a):
        fake.calls.append(a)
        return 0

    for f in (c.fake, fake):
        for name in ("attention", "attention_shared"):
            monkeypatch.setattr(f, name, launched, raising=False)
    calls[call]()
    assert inside and inside[0] in alive  # what the launch was given was still there
    gc.collect()
    assert all(t() is None for t in tensors)  # and is the allocator's afterwards
    assert len(paged._workspaces) + len(paged._captured) == 1
