"""Build ``libppow.so`` (sm_100a only) in-tree with nvcc.  ``python -m paper_2605_14978_b200.build``."""
from __future__ import annotations

import concurrent.futures
import glob
import os
import shutil
import subprocess
import sys
import tempfile
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libppow.so")
LIB_CHECKED = os.path.join(HERE, "libppow_checked.so")   # the same sources with -DPPOW_CHECKED (bounds-checked build)
LIB_TIMELINE = os.path.join(HERE, "libppow_timeline.so")  # ... with -DPPOW_TIMELINE (per-warp timeline of the row kernel)
CALLS = os.path.join(HERE, "_calls.so")                 # csrc/ppow_calls.cpp: one call from Python per training-end operator
ROOT = os.path.dirname(HERE)


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def is_stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(f) > t for f in _deps())


def _torch_mark() -> str:
    """What _calls.so carries to say which torch it was built against."""
    import torch
    return "ppow_calls for torch " + torch.__version__


def calls_are_stale() -> bool:
    """Missing, older than its sources, or built against another torch than the installed one."""
    deps = [os.path.join(CSRC, "ppow_calls.cpp"), os.path.join(ROOT, "include", "ppow.h")]
    if not os.path.exists(CALLS) or any(os.path.getmtime(f) > os.path.getmtime(CALLS) for f in deps):
        return True
    with open(CALLS, "rb") as f:
        return _torch_mark().encode() + b"\0" not in f.read()


def build_calls(force: bool = False) -> str:
    """Compile the extension module that marshals the training-end calls, against the torch that is installed."""
    if not force and not calls_are_stale():
        return CALLS
    import sysconfig
    import torch
    at = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(shutil.which(os.environ.get("NVCC", "nvcc")) or "/usr/local/cuda/bin/nvcc"))
    tmp = CALLS + ".tmp.%d.%d" % (os.getpid(), threading.get_ident())
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), '-DPPOW_TORCH_MARK="%s"' % _torch_mark(),
           "-I" + os.path.join(at, "include"), "-I" + os.path.join(at, "include", "torch", "csrc", "api", "include"),
           "-I" + os.path.join(cuda, "include"), "-I" + sysconfig.get_path("include"), os.path.join(CSRC, "ppow_calls.cpp"), "-o", tmp,
           "-L" + os.path.join(at, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cuda", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stderr)
    os.replace(tmp, CALLS)
    return CALLS


def build(force: bool = False, verbose: bool = False, checked: bool = False, timeline: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared library for sm_100a.  ``checked``: the bounds-checked
    build (every kernel-computed index tested before use, failures counted and skipped, never trapped)."""
    lib = LIB_CHECKED if checked else LIB_TIMELINE if timeline else LIB
    if force or is_stale(lib):
        _build_library(lib, verbose, checked, timeline)
    build_calls(force and lib == LIB)        # behind the library, which does without it
    return lib


def _build_library(lib: str, verbose: bool, checked: bool, timeline: bool) -> None:
    nvcc = os.environ.get("NVCC", "nvcc")
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC"]
    flags += ["-Xptxas", "-v"] if verbose else []
    flags += ["-DPPOW_CHECKED"] if checked else ["-DPPOW_TIMELINE"] if timeline else []

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose:
            sys.stderr.write(res.stderr)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stderr)

    with tempfile.TemporaryDirectory(prefix="ppow_build_") as objects:       # one compiler per source file, side by side
        outs = [os.path.join(objects, os.path.basename(src) + ".o") for src in sources()]
        with concurrent.futures.ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:
            list(pool.map(lambda so: run([nvcc] + flags + ["-c", so[0], "-o", so[1]]), zip(sources(), outs)))
        tmp = lib + ".tmp.%d" % os.getpid()
        run([nvcc] + flags + ["-shared", "-o", tmp] + outs)
    os.replace(tmp, lib)


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build(force=True, checked=True))
    print(build(force=True, timeline=True))
