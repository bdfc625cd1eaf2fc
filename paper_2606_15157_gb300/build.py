"""Build the CUDA libraries in-tree (``paper_2606_15157_gb300/lib``) for sm_103a.

``libkvev.so``        the eviction library (C ABI of ``include/kvev.h``);
``libkvev_synth.so``  the device-side synthetic input generator
                      (C ABI of ``include/kvev_synth.h``);
``kvev_paged_bind.so``, ``kvev_paged_q8_bind.so``
                      the extension modules through which ``paged.py`` calls ``libkvev.so``
                      with torch tensors (host code only; left out where torch is not installed).

Translation units are compiled in parallel with nvcc, then linked; a unit is
rebuilt only when it or a header it includes changed, the extension modules also
for another torch, Python or compiler.  What fails to build of the extension modules
is raised when the C libraries are there.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
OBJDIR = os.path.join(LIBDIR, "obj")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include")]

LIBS = {
    "libkvev.so": ["api.cu", "score.cu", "h2o_full.cu", "select.cu", "gather.cu", "decode.cu", "planner.cu",
                   "paged.cu", "paged_attn.cu", "paged_shared.cu", "paged_q8.cu", "paged_q8_attn.cu"],
    "libkvev_synth.so": ["synth.cu"],
}


BIND = "kvev_paged_bind.so"
BINDS = {BIND: "paged_bind.cpp", "kvev_paged_q8_bind.so": "paged_q8_bind.cpp"}
CXX = os.environ.get("CXX", "g++")


def _torch_dir() -> str | None:
    import importlib.util
    spec = importlib.util.find_spec("torch")  # (without importing it)
    return None if spec is None else os.path.dirname(spec.origin)


def _bind_flags() -> tuple[list[str], list[str]]:
    """(compiler, linker) flags of the extension modules: Python's, torch's and CUDA's headers and libraries."""
    torch_dir = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(NVCC))
    libs = os.path.join(torch_dir, "lib")
    return (["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", os.path.join(torch_dir, "include"),
             "-I", os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
             "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"), "-I", os.path.join(ROOT, "include")],
            ["-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{libs}",
             "-L", os.path.join(cuda, "lib64"), "-lcudart",
             "-L", LIBDIR, "-l:libkvev.so", "-Wl,-rpath,$ORIGIN"])


def _run(cmd: list[str], what: str):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")


def _bind_made_with() -> str:
    """What an extension module's object depends on beside the sources."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        return "\n".join([CXX, *_bind_flags()[0], sys.version, f.read()])


def _compile_bind(name: str) -> str:
    src, obj = os.path.join(CSRC, name), os.path.join(OBJDIR, name + ".o")
    made, want = obj + ".made_with", _bind_made_with()
    same = os.path.exists(made) and open(made).read() == want
    if not same or _stale(obj, [src] + _headers()):
        tmp = obj + f".tmp{os.getpid()}"
        _run([CXX, *_bind_flags()[0], "-c", src, "-o", tmp], f"{CXX} failed for {src}")
        os.replace(tmp, obj)
        with open(made, "w") as f:
            f.write(want)
    return obj


def _headers():
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _stale(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src: str, extra: list[str]) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    if _stale(obj, [src] + _headers()):
        tmp = obj + f".tmp{os.getpid()}"
        cmd = [NVCC, *ARCH, *FLAGS, *extra, "-c", src, "-o", tmp]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, obj)
    return obj


def build(verbose: bool = False, extra: list[str] | None = None) -> dict[str, str]:
    """Compile every library; returns {name: path} of those that there are."""
    os.makedirs(OBJDIR, exist_ok=True)
    extra = list(extra or [])
    out = {}
    srcs = sorted({s for v in LIBS.values() for s in v})
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 4)) as ex:
        binds = {lib: ex.submit(_compile_bind, src) for lib, src in BINDS.items()} if _torch_dir() else None
        objs = dict(zip(srcs, ex.map(lambda s: _compile(os.path.join(CSRC, s), extra), srcs)))
    for lib, units in LIBS.items():
        path = os.path.join(LIBDIR, lib)
        deps = [objs[u] for u in units]
        if _stale(path, deps):
            tmp = path + f".tmp{os.getpid()}"
            cmd = [NVCC, *ARCH, "-shared", "-o", tmp, *deps]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"link failed for {lib}:\n{r.stdout}\n{r.stderr}")
            os.replace(tmp, path)
        if verbose:
            print("built", path)
        out[lib] = path
    if binds is None:
        if verbose:
            print("not built:", *BINDS, "(torch is not installed)")
        return out
    for lib, bind in binds.items():
        bind_obj = bind.result()
        path = os.path.join(LIBDIR, lib)
        if _stale(path, [bind_obj, out["libkvev.so"]]):
            tmp = path + f".tmp{os.getpid()}"
            _run([CXX, "-shared", "-o", tmp, bind_obj, *_bind_flags()[1]], f"link failed for {lib}")
            os.replace(tmp, path)
        if verbose:
            print("built", path)
        out[lib] = path
    return out


if __name__ == "__main__":
    build(verbose=True)
