"""What build() makes when the extension module cannot be made, and when it is made anew (no GPU needed)."""
import os

import pytest


@pytest.fixture()
def fresh(tmp_path, monkeypatch):
    """The build module with an empty library folder and the objects that are there."""
    from paper_2606_15157_gb300 import build
    build.build()
    monkeypatch.setattr(build, "LIBDIR", str(tmp_path))
    return build, tmp_path


def test_without_torch_the_c_libraries_are_built(fresh, monkeypatch):
    import importlib.util
    build, lib = fresh
    real = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else real(name, *a))
    os.remove(os.path.join(build.OBJDIR, "paged_bind.cpp.o"))
    made = build.build()
    assert set(made) == set(build.LIBS)
    assert all(os.path.exists(lib / name) for name in build.LIBS) and not os.path.exists(lib / build.BIND)


def test_a_failing_host_compiler_stops_after_the_c_libraries(fresh, monkeypatch):
    build, lib = fresh
    monkeypatch.setattr(build, "CXX", "false")
    os.remove(os.path.join(build.OBJDIR, "paged_bind.cpp.o"))
    with pytest.raises(RuntimeError, match="paged_bind"):
        build.build()
    assert all(os.path.exists(lib / name) for name in build.LIBS)


def test_the_extension_is_made_anew_for_another_torch_or_python(fresh, monkeypatch):
    build, _ = fresh
    build.build()
    obj = os.path.join(build.OBJDIR, "paged_bind.cpp.o")
    at = os.path.getmtime(obj)
    build.build()
    assert os.path.getmtime(obj) == at
    flags, links = build._bind_flags()
    monkeypatch.setattr(build, "_bind_flags", lambda: (flags + ["-DKVEV_OTHER_TORCH"], links))
    build.build()
    assert os.path.getmtime(obj) > at
