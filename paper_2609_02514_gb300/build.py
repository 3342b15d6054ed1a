"""Builds libacespec.so in this package directory from csrc/*.cu for sm_103a.

Each translation unit is compiled in parallel with nvcc, then linked into one
shared library (CUDA runtime linked statically).  Re-running is a no-op when
the library is newer than every source.  build(checked=True) makes the
checked test build instead, libacespec_checked.so (-DACES_CHECKED: every
kernel records out-of-range indices instead of using them).
The native half of the Python binding (csrc/binding.cpp, against torch's
headers) is compiled alongside with the host compiler, into a file named
after Python's and torch's versions, where there are torch, Python's headers
and a C++ compiler.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libacespec.so")
LIB_CHECKED = os.path.join(HERE, "libacespec_checked.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
BINDING_SRC = os.path.join(CSRC, "binding.cpp")
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2"]


def binding_path(torch_version: str) -> str:
    """The binding for this Python and a version of torch: built against one of each, it must not be
    loaded by another."""
    return os.path.join(HERE, f"_binding.{sys.implementation.cache_tag}.torch-{torch_version}.so")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libacespec.so")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + [
        os.path.join(ROOT, "include", "acespec.h")]


def up_to_date(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(p) <= t for p in _deps())


def _no_binding(why: str) -> None:
    print(f"the binding (the Python calls of the 4-bit cache) is not built: {why}", file=sys.stderr)


def _start_binding(force: bool):
    """The compiler at work on the binding (its command, process and result), or None when it is newer than
    its sources, or when it cannot be built here: a C caller needs libacespec.so alone."""
    import sysconfig
    try:
        import torch
    except Exception as e:  # not installed, or not loadable on this machine
        return _no_binding(f"torch cannot be imported ({e})")
    path = binding_path(torch.__version__)
    deps = [BINDING_SRC, os.path.join(ROOT, "include", "acespec.h")]
    if not force and os.path.exists(path) and all(os.path.getmtime(p) <= os.path.getmtime(path) for p in deps):
        return None
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        return _no_binding("no C++ compiler")
    headers = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(headers, "Python.h")):
        return _no_binding(f"no Python.h in {headers}")
    base, abi = os.path.dirname(torch.__file__), int(torch.compiled_with_cxx11_abi())
    inc = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), headers]
    cmd = [cxx, "-std=c++17", "-O1", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={abi}"]
    cmd += [f"-I{i}" for i in inc] + ["-o", path + f".tmp{os.getpid()}", BINDING_SRC, "-L" + os.path.join(base, "lib"),
                                      "-ltorch_python", "-ltorch_cpu", "-lc10"]
    return cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT), path


def _finish_binding(started) -> None:
    """Waits for the compiler; an error of its own is raised when the library is there."""
    if started is None:
        return
    cmd, p, path = started
    out, _ = p.communicate()
    if p.returncode != 0:
        raise RuntimeError("the binding does not compile: " + " ".join(cmd) + "\n" + out.decode(errors="replace"))
    os.replace(cmd[cmd.index("-o") + 1], path)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    lib = LIB_CHECKED if checked else LIB
    binding = _start_binding(force)
    if not force and up_to_date(lib):
        _finish_binding(binding)
        return lib
    nvcc = _nvcc()
    bdir = os.path.join(HERE, "_build_checked" if checked else "_build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    objs = []
    for src in _sources():
        obj = os.path.join(bdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc] + ARCH + FLAGS + (["-DACES_CHECKED"] if checked else []) + ["-c", src, "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    for cmd, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd) + "\n" + out.decode(errors="replace"))
        if verbose and out:
            sys.stdout.write(out.decode(errors="replace"))
    tmp = lib + f".tmp{os.getpid()}"
    link = [nvcc] + ARCH + ["-shared", "-o", tmp] + objs
    r = subprocess.run(link, capture_output=True)
    if r.returncode != 0:
        raise RuntimeError("link failed: " + " ".join(link) + "\n" + r.stdout.decode() + r.stderr.decode())
    os.replace(tmp, lib)
    _finish_binding(binding)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, checked="--checked" in sys.argv))
